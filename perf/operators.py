"""Serving operators on a compacted K/V cache, as a program that decodes behind the compression runs them.

After the prefill every request holds the pages that compact_kv left it.  From then on a serving step

  pages    brings the block tables in line with the requests' lengths (pages that a shrunken or finished request no longer
           needs go back to the free list, growing requests get theirs) and lists the slot of every new token,
  append   writes the new tokens' keys and values to those slots,
  decode   lets one new token per request attend to everything the request holds, perhaps writing its own key and value
           on the way.

A case is a dict with "op" and
  pages:  batch, lo / hi (lengths before the call, spread evenly over their logarithm; hi = 0: empty tables), mode
          ("step": every request grows by one token; "shrink": lengths fall to about half; "admit": new lengths
          from new_lo / new_hi; "mixed": finished, shrunken, growing and unchanged requests), page, idle (share of
          batch places without a request)
  append: tokens, kv_heads, head_dim, page, dtype, layout, skip (share of rows without a slot)
  decode: batch, heads, kv_heads, head_dim, lo / hi (keys per request), page, dtype, layout, new (the token's own key and
          value come along), idle
layout: "head_major" ([page, head, row, channel] in memory) or "token_major" ([page, row, head, channel]).
"""
from __future__ import annotations

import math

import torch

own = False

SCRATCH = 32 << 20


def _decode(name, batch, heads, kv_heads, head_dim, lo, hi, page=16, dtype="bf16", layout="head_major", new=True, idle=0.0):
    return dict(name=name, op="decode", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, lo=lo, hi=hi,
                page=page, dtype=dtype, layout=layout, new=new, idle=idle)


def _append(name, tokens, kv_heads, head_dim, page=16, dtype="bf16", layout="head_major", skip=0.0):
    return dict(name=name, op="append", tokens=tokens, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype,
                layout=layout, skip=skip)


def _pages(name, batch, mode, lo, hi, new_lo=0, new_hi=0, page=16, idle=0.0):
    return dict(name=name, op="pages", batch=batch, mode=mode, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, page=page,
                idle=idle)


def listed():
    return [
        # one interactive request of a 7B model behind one halved image: latency of a layer's attention
        _decode("one_request", 1, 32, 32, 128, 404, 404),
        # a small chat batch, grouped heads, ragged lengths
        _decode("chat_batch", 16, 32, 8, 128, 150, 1500),
        # two video conversations with very long caches, seven query heads a key head, no new token of their own
        _decode("long_cache", 2, 28, 4, 128, 60001, 131072, page=64, new=False),
        # many image conversations on a 13B model without grouped heads
        _decode("wide_batch", 48, 40, 40, 128, 301, 1399, page=32, layout="token_major"),
        # a full engine: lengths from a few tokens to thousands, some places of the batch without a request
        _decode("full_engine", 96, 32, 8, 128, 37, 8192, idle=0.1),
        # heads of 64
        _decode("narrow_heads", 24, 32, 8, 64, 90, 2000, page=16),
        # single precision storage and arithmetic
        _decode("single_precision", 4, 8, 8, 128, 211, 777, dtype="fp32", new=False),
        # the new rows of a decoding batch
        _append("step_rows", 64, 8, 128, skip=0.1),
        # the new rows of a prefill of several prompts
        _append("prefill_rows", 32768, 8, 128, layout="token_major"),
        # the tables of a decoding batch: most steps move a page for one request in sixteen
        _pages("decode_step", 256, "step", 100, 4000, idle=0.1),
        # behind an in-place compaction: every request gives pages back
        _pages("after_compaction", 64, "shrink", 400, 6000),
        # prompts of a whole batch are admitted at once
        _pages("admit_prompts", 128, "admit", 0, 0, 500, 8000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mean(lo, hi):
    """Mean of what is spread evenly over the logarithm between lo and hi."""
    return float(lo) if hi <= lo else (hi - lo) / math.log(hi / lo)


def draw(rng):
    """A case of the ranges above: 1 to 128 requests of 1 to 131072 keys, 1 to 40 key heads of 32 to 256 channels shared by
    up to 16 query heads, pages of 1 to 256 rows; up to 32768 rows appended; tables of 4 to 1024 requests."""
    limit = work(next(c for c in listed() if c["name"] == "full_engine"))["bytes"]
    kind = rng.random()
    page = rng.choice([16, 16, 16, 32, 64, 128, 256, 1, 7, 24])
    layout = rng.choice(["head_major", "head_major", "token_major"])
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    while True:
        if kind < 0.6:
            kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 16, 32, 40])
            hi, batch = _log_int(rng, 16, 131072), _log_int(rng, 1, 128)
            case = _decode(None, batch, kv_heads * rng.choice([1, 1, 2, 4, 4, 7, 8, 16]), kv_heads,
                           rng.choice([128, 128, 128, 64, 64, 96, 80, 256, 32]), _log_int(rng, 1, hi), hi, page, dtype,
                           layout, rng.random() < 0.6, rng.choice([0.0, 0.0, 0.1, 0.3]) if batch >= 8 else 0.0)
            if case["heads"] > 128 or page == 1 and hi > 20000 or case["batch"] * hi > 4000000:
                continue
            padded = 4.0 * case["batch"] * hi * kv_heads * case["head_dim"]
            if padded > 4e9 or padded * case["heads"] / kv_heads > 3e10:   # the plain form fills every row up to the longest
                continue
        elif kind < 0.78:
            case = _append(None, _log_int(rng, 1, 32768), rng.choice([1, 2, 4, 8, 8, 16, 32]),
                           rng.choice([128, 128, 64, 96, 80, 256, 8]), page, dtype, layout, rng.choice([0.0, 0.1, 0.5]))
        else:
            mode = rng.choice(["step", "step", "shrink", "admit", "mixed"])
            hi = 0 if mode == "admit" else _log_int(rng, 16, 16000)
            new_hi = _log_int(rng, 16, 8000) if mode in ("admit", "mixed") else 0
            case = _pages(None, _log_int(rng, 4, 1024), mode, _log_int(rng, 1, hi) if hi else 0, hi,
                          _log_int(rng, 1, new_hi) if new_hi else 0, new_hi, page, rng.choice([0.0, 0.1, 0.3]))
            if case["batch"] * max(hi, new_hi) > 2000000:
                continue
        case.pop("name")
        if work(case)["bytes"] <= limit:
            return case


def work(case):
    """Decode: every key and value that a request holds read once, the query and the answer; two products.  Append: every row
    read and written once.  Pages: lengths, the page numbers that change hands, and the slots."""
    el = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "decode":
        b, h, hk, dh = (case[k] for k in ("batch", "heads", "kv_heads", "head_dim"))
        live = b * (1 - case["idle"])
        keys = live * _mean(case["lo"], case["hi"])
        n_bytes = 2 * keys * hk * dh * el + 2 * b * h * dh * el + 4 * b * h + 4 * keys / case["page"]
        if case["new"]:
            n_bytes += 2 * live * hk * dh * el
        return {"bytes": n_bytes, "flops": 4.0 * keys * h * dh}
    if case["op"] == "append":
        rows = case["tokens"] * (1 - case["skip"])
        return {"bytes": 4.0 * rows * case["kv_heads"] * case["head_dim"] * el + 8 * case["tokens"], "flops": 0.0}
    b, page = case["batch"] * (1 - case["idle"]), case["page"]
    rows = case["batch"] if case["mode"] == "step" else _budget(case)
    held, new = _mean(case["lo"], case["hi"]) if case["hi"] else 0.0, _mean(case["new_lo"], case["new_hi"]) if case["new_hi"] else 0.0
    moved = {"step": 1.0 / page, "shrink": held / 2 / page, "admit": new / page + 0.5,
             "mixed": (new / 4 + held / 2) / page}[case["mode"]]
    return {"bytes": 16.0 * case["batch"] + 8 * b * moved + 8 * rows, "flops": 0.0}


# ----------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _lengths(n, lo, hi, gen):
    """[n] int64 lengths, evenly over their logarithm."""
    u = torch.rand((n,), generator=gen, device="cuda", dtype=torch.float64)
    v = torch.exp(math.log(max(lo, 1)) + u * math.log(max(hi, 1) / max(lo, 1)))
    return v.round().long().clamp(min=lo, max=hi)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _budget(case):
    """Rows of a call's slot map: the step's token budget, a quarter above what is expected."""
    share = {"admit": 1.0, "mixed": 0.5}.get(case["mode"], 0.0)
    return 64 + int(1.25 * share * case["batch"] * (_mean(case["new_lo"], case["new_hi"]) + 1)) if share else 1


def _pool(case, n_pages, gen):
    """A page pool [n_pages, kv_heads, page, head_dim] in the case's layout."""
    hk, dh, page = case["kv_heads"], case["head_dim"], case["page"]
    if case["layout"] == "token_major":
        return torch.randn((n_pages, page, hk, dh), generator=gen, device="cuda", dtype=_dtype(case)).permute(0, 2, 1, 3)
    return torch.randn((n_pages, hk, page, dh), generator=gen, device="cuda", dtype=_dtype(case))


def _tables(blocks, width, n_pages, gen):
    """Block table [B, width] whose row b holds blocks[b] of n_pages pages (the rest: 0), all different, and the pages left."""
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    first = blocks.cumsum(0) - blocks
    j = torch.arange(width, device="cuda")
    at = (first[:, None] + j[None, :]).clamp(max=n_pages - 1)
    table = torch.where(j[None, :] < blocks[:, None], order[at], torch.zeros((), dtype=torch.long, device="cuda"))
    return table.int().contiguous(), order[int(blocks.sum()):].int()


def prepare(case, seed):
    gen = _generator(seed)
    page = case["page"]
    s = dict(case=case, scratch=torch.empty((SCRATCH,), dtype=torch.uint8, device="cuda"))
    if case["op"] == "decode":
        b, h, hk, dh = (case[k] for k in ("batch", "heads", "kv_heads", "head_dim"))
        n = _lengths(b, case["lo"], case["hi"], gen)
        n[torch.rand((b,), generator=gen, device="cuda") < case["idle"]] = 0
        blocks = (n + page - 1) // page
        width = -(-case["hi"] // page)
        n_pages = b * width + 3                            # the engine's pool, of which the requests hold a part
        s["table"], _ = _tables(blocks, width, n_pages, gen)
        s.update(n_keys=n.int(), k_cache=_pool(case, n_pages, gen), v_cache=_pool(case, n_pages, gen), k_new=None, v_new=None)
        s["q"] = 2 * torch.randn((b, h, dh), generator=gen, device="cuda").to(_dtype(case))
        if case["new"]:
            s["k_new"], s["v_new"] = (torch.randn((b, hk, dh), generator=gen, device="cuda").to(_dtype(case)) for _ in range(2))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((b, h), device="cuda", dtype=torch.float32)
    elif case["op"] == "append":
        t, hk, dh = case["tokens"], case["kv_heads"], case["head_dim"]
        n_pages = -(-t // page) + 2
        # requests of some length each: runs of slots inside a page follow one another, pages come in any order
        order = torch.randperm(n_pages, generator=gen, device="cuda")
        at = torch.arange(t, device="cuda") + page // 2
        slot = order[at // page] * page + at % page
        slot[torch.rand((t,), generator=gen, device="cuda") < case["skip"]] = -1
        s.update(slot_map=slot, k_cache=_pool(case, n_pages, gen), v_cache=_pool(case, n_pages, gen))
        s["k_new"], s["v_new"] = (torch.randn((t, hk, dh), generator=gen, device="cuda").to(_dtype(case)) for _ in range(2))
    else:
        b, mode = case["batch"], case["mode"]
        zero = torch.zeros((b,), dtype=torch.long, device="cuda")
        held = _lengths(b, case["lo"], case["hi"], gen) if case["hi"] else zero
        new = _lengths(b, case["new_lo"], case["new_hi"], gen) if case["new_hi"] else zero
        idle = torch.rand((b,), generator=gen, device="cuda") < case["idle"]
        add, stride, which = 0, 0, torch.randint(0, 4, (b,), generator=gen, device="cuda")
        if mode == "step":                                 # the new length is the old one and a token
            base, add, stride = held, 1, 1
        elif mode == "shrink":                             # prompt rows and what the compaction left of the vision rows
            add = min(64, case["lo"])
            base = (held - add) // 2
        elif mode == "admit":
            base = new
        else:
            base = torch.where(which == 0, held // 2, torch.where(which == 1, held + new, torch.where(which == 2, held + 1, held)))
            idle = idle | (torch.rand((b,), generator=gen, device="cuda") < 0.1)
        if mode == "mixed":                                # requests that finish give everything back
            base = torch.where(idle, torch.full_like(base, -1), base)
        else:
            held, base = torch.where(idle, zero - 1, held), torch.where(idle, zero - 1, base)
        have = (held.clamp(min=0) + page - 1) // page
        most = case["hi"] + case["new_hi"] + 1
        want = torch.where(base < 0, zero, base + add)
        grow = ((want + page - 1) // page - have).clamp(min=0)
        width = -(-most // page)
        n_pages = b * width + 5
        table, free = _tables(have, width, n_pages, gen)
        stack = torch.zeros((n_pages,), dtype=torch.int32, device="cuda")
        stack[:free.numel()] = free
        spare = free.numel()
        if mode == "mixed" and which[0] >= 2:              # other users of the pool hold what half of the requests ask for
            spare = min(spare, max(1, int(grow.sum()) // 2))
        rows = b if stride else _budget(case)
        i32 = dict(dtype=torch.int32, device="cuda")
        s.update(held=held.int(), seq_len=base.int(), add=add, stride=stride, table=table, free=stack,
                 n_free=torch.tensor([spare], **i32), len_out=torch.zeros((b,), **i32), n_free_out=torch.zeros((1,), **i32),
                 slot_map=torch.zeros((rows,), dtype=torch.int64, device="cuda"), slot_start=torch.zeros((b + 1,), **i32))
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------------ plain forms

def _plain_decode(s):
    case, q, n = s["case"], s["q"], s["n_keys"].long()
    page, (b, h, dh), hk = case["page"], q.shape, case["kv_heads"]
    if case["new"]:                                        # the token's own row is the last that it sees
        last = (n - 1).clamp(min=0)
        at = s["table"].long().gather(1, (last // page)[:, None])[:, 0]
        live = n > 0
        s["k_cache"][at[live], :, last[live] % page] = s["k_new"][live]
        s["v_cache"][at[live], :, last[live] % page] = s["v_new"][live]
    rows = s["table"].long()

    def gathered(cache):                                   # [B, Hk, keys, dh] in 32 bits
        return cache[rows].permute(0, 2, 1, 3, 4).reshape(b, hk, -1, dh).float()

    k = gathered(s["k_cache"])
    seen = torch.arange(k.shape[2], device="cuda")[None, :] < n[:, None]
    logits = torch.matmul(q.float().view(b, hk, h // hk, dh), k.transpose(2, 3)) / math.sqrt(dh)
    del k
    logits = torch.where(seen[:, None, None, :], logits, torch.full((), -math.inf, device="cuda"))
    top = logits.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(logits - top)
    total = p.sum(dim=3, keepdim=True)
    v = torch.where(seen[:, None, :, None], gathered(s["v_cache"]), torch.zeros((), device="cuda"))
    out = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + torch.log(total)).view(b, h)
    result = [out.view(b, h, dh).to(q.dtype), lse]
    return result + [s["k_cache"], s["v_cache"]] if case["new"] else result


def _plain_append(s):
    page, keep = s["case"]["page"], s["slot_map"] >= 0
    slot = s["slot_map"][keep]
    s["k_cache"][slot // page, :, slot % page] = s["k_new"][keep]
    s["v_cache"][slot // page, :, slot % page] = s["v_new"][keep]
    return [s["k_cache"], s["v_cache"]]


def _plain_pages(s):
    page, table, stack = s["case"]["page"], s["table"].long(), s["free"].long()
    held, base, n_free = s["held"].long().clamp(min=0), s["seq_len"].long(), s["n_free"].long()
    width, dev = table.shape[1], "cuda"
    active = base >= 0
    want = torch.where(active, base + s["add"], torch.zeros_like(base))
    have, need = (held + page - 1) // page, (want + page - 1) // page
    gone, grow = (have - need).clamp(min=0), (need - have).clamp(min=0)
    gone_to, grow_to = gone.cumsum(0), grow.cumsum(0)
    on_stack = n_free + gone_to[-1:]
    granted = grow_to <= on_stack
    taken = torch.where(granted, grow, torch.zeros_like(grow))
    left = on_stack - taken.sum()
    j = torch.arange(width, device=dev)[None, :]
    # released pages lie above the free ones, in the order of the requests; the last entry takes what is none
    place = n_free + (gone_to - gone)[:, None] + j - need[:, None]
    released = (j >= need[:, None]) & (j < have[:, None])
    piled = torch.cat([stack, stack.new_zeros(1)])
    piled = piled.scatter(0, torch.where(released, place, torch.full_like(place, stack.numel())).reshape(-1), table.reshape(-1))
    # the k-th page that is asked for comes from the top
    k = (grow_to - grow)[:, None] + j - have[:, None]
    gets = (j >= have[:, None]) & (j < need[:, None]) & granted[:, None]
    table = torch.where(gets, piled[(on_stack - 1 - k).clamp(min=0, max=stack.numel())], table)
    at = torch.arange(stack.numel(), device=dev)
    stack = torch.where(at < left, piled[:-1], stack)
    length = torch.where(active, torch.where(granted | (grow == 0), want, held), base)
    fresh = (want - held).clamp(min=0)
    start = torch.cat([fresh.new_zeros(1), fresh.cumsum(0)])
    t = torch.arange(s["slot_map"].numel(), device=dev)
    if s["stride"]:
        b, i = t // s["stride"], t % s["stride"]
    else:
        b = torch.searchsorted(start[1:], t, right=True).clamp(max=held.numel() - 1)
        i = t - start[b]
    p = held[b] + i
    slot = table[b, (p // page).clamp(max=width - 1)] * page + p % page
    slot = torch.where((i < fresh[b]) & (granted | (grow == 0))[b], slot, torch.full_like(slot, -1))
    return [length.int(), table.int(), stack.int(), left.int(), slot, start.int()]


def run(s):
    case = s["case"]
    if not own:
        return {"decode": _plain_decode, "append": _plain_append, "pages": _plain_pages}[case["op"]](s)
    import paper_2605_00789_b200 as L
    if case["op"] == "decode":
        L.decode_attention(s["q"], s["k_cache"], s["v_cache"], s["n_keys"], s["out"], block_table=s["table"], lse=s["lse"],
                           k_new=s["k_new"], v_new=s["v_new"], workspace=s["scratch"])
        return [s["out"], s["lse"], s["k_cache"], s["v_cache"]] if case["new"] else [s["out"], s["lse"]]
    if case["op"] == "append":
        L.append_kv(s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["slot_map"])
        return [s["k_cache"], s["v_cache"]]
    L.assign_pages(s["seq_len"], s["table"], s["free"], s["n_free"], page_size=case["page"], add=s["add"], held=s["held"],
                   seq_len_out=s["len_out"], n_free_out=s["n_free_out"], slot_map=s["slot_map"], slot_start=s["slot_start"],
                   slot_stride=s["stride"], workspace=s["scratch"])
    return [s["len_out"], s["table"], s["free"], s["n_free_out"], s["slot_map"], s["slot_start"]]


# ------------------------------------------------------------------------------------------------------- definitions

def _exact_decode(s):
    """softmax(q K^T / sqrt(dh)) V of every request by itself; the caches hold moved values only."""
    case, dh = s["case"], s["case"]["head_dim"]
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["n_keys"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // case["page"])].long()
        k, v = (c[pages].transpose(0, 1).reshape(case["kv_heads"], -1, dh)[:, :n].double() for c in (s["k_cache"], s["v_cache"]))
        if case["new"]:
            k[:, n - 1], v[:, n - 1] = s["k_new"][b].double(), s["v_new"][b].double()
        q = s["q"][b].double().view(case["kv_heads"], group, dh)
        logits = torch.einsum("hgd,hnd->hgn", q, k) * dh ** -0.5
        lse[b] = torch.logsumexp(logits, dim=2).reshape(-1)
        out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(logits, dim=2), v).reshape(-1, dh)
    return [out, lse, None, None] if case["new"] else [out, lse]


def _exact_append(s):
    page, kept = s["case"]["page"], []
    slots = s["slot_map"].tolist()
    rows = [t for t, slot in enumerate(slots) if slot >= 0]
    for cache, new in ((s["k_cache"], s["k_new"]), (s["v_cache"], s["v_new"])):
        c = cache.double()
        flat = c.transpose(1, 2).reshape(-1, *new.shape[1:])      # slot by slot
        flat[torch.tensor([slots[t] for t in rows], dtype=torch.long, device="cuda")] = new[rows].double()
        kept.append(flat.view(c.shape[0], page, *new.shape[1:]).transpose(1, 2).contiguous())
    return kept


def _exact_pages(s):
    """One request after the other, with a list as the stack of free pages."""
    page, table = s["case"]["page"], s["table"].tolist()
    held, base = [max(v, 0) for v in s["held"].tolist()], s["seq_len"].tolist()
    memory = s["free"].tolist()
    stack = memory[:int(s["n_free"])]
    want = [v + s["add"] if v >= 0 else 0 for v in base]
    pages = lambda n: -(-n // page)  # noqa: E731
    for b in range(len(base)):
        stack += table[b][pages(want[b]):pages(held[b])]
    length, asked, room, slots, start = [], 0, len(stack), [], [0]
    for b in range(len(base)):
        more, fresh = pages(want[b]) - pages(held[b]), max(want[b] - held[b], 0)
        asked += max(more, 0)
        given = more <= 0 or asked <= room
        for j in range(max(more, 0) if given else 0):
            table[b][pages(held[b]) + j] = stack.pop()
        length.append(base[b] if base[b] < 0 else want[b] if given else held[b])
        mine = [table[b][p // page] * page + p % page if given else -1 for p in range(held[b], held[b] + fresh)]
        if s["stride"]:
            mine = (mine + [-1] * s["stride"])[:s["stride"]]
        slots += mine
        start.append(start[-1] + fresh)
    slots = (slots + [-1] * s["slot_map"].numel())[:s["slot_map"].numel()]
    memory[:len(stack)] = stack
    as_int = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return [as_int(length), as_int(table), as_int(memory), as_int([len(stack)]), torch.tensor(slots), as_int(start)]


def exact(case, seed):
    s = prepare(case, seed)
    return {"decode": _exact_decode, "append": _exact_append, "pages": _exact_pages}[case["op"]](s)
