"""The serving calls where one meets another, and at edges of their arguments: against the oracle, with the tolerances of
tests/test_serving.py (its head derives them)."""
import ctypes as C
import math
import os
import re
import subprocess

import numpy as np
import pytest

import __graft_entry__ as entry
from oracle import serving as O
from tests.test_kernel_units import _run
from tests.test_serving import Decode, _call_pages, _decode_args, _f64, _i32, _random, _random_pages

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    entry.build()
    import paper_2605_00789_b200 as pkg
    return pkg


# ------------------------------------------------------------------------------------------------------ without a GPU

def _documented_loop():
    """The body of the decoding loop that the users' page shows."""
    block = re.search(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S).group(1)
    body = block[block.index("for step in range(n):"):].split("\n", 1)[1]
    return "\n".join(line[4:] for line in body.splitlines() if line.startswith("    "))


def test_the_documented_loop_hands_the_slots_on():
    calls = [c for c in re.split(r"\n(?=\S)", _documented_loop()) if c]
    assert [c.split("(")[0] for c in calls] == ["L.assign_pages", "L.decode_attention"]
    assert all("slot_map=slots" in c and "status=status" in c for c in calls) and "slot_stride=1" in calls[0]


@pytest.mark.parametrize("kw", [dict(slot_map=0x9000), dict(k_new=0x7000, v_new=0x8000, slot_map=0x9004)])
def test_decode_attention_refuses_a_slot_map(L, kw):
    """Without new rows, and where it is not aligned."""
    assert L.library().lightkv_decode_attention(C.byref(_decode_args(L, **kw))) == -1


def test_decode_attention_refuses_a_negative_bound(L):
    for kw in (dict(max_keys=-1), dict(page_size=0, max_keys=100, key_bound=-1), dict(key_bound=-1)):
        assert L.library().lightkv_decode_attention(C.byref(_decode_args(L, **kw))) == -1


def test_oracle_new_row():
    k, v = np.zeros((2, 3, 4)), np.ones((2, 3, 4))
    row = np.full((2, 4), 5.0)
    kk, vv = O.with_new_row(k, v, row, 2 * row)
    assert (kk[:, 2] == 5).all() and (vv[:, 2] == 10).all() and (kk[:, :2] == 0).all() and (k == 0).all()
    kk, vv = O.with_new_row(k, v, row, row, -1)
    assert (kk == k).all() and (vv == v).all()


def _kernel_body(name):
    """The text of a kernel of the attention, without comments."""
    text = open(os.path.join(entry.CSRC, "lightkv_decode.cu")).read()
    text = text[text.index(name + "(const __grid_constant__"):]
    return re.sub(r"//.*", "", text[:text.index("\n}\n")])


def test_no_cta_is_counted_on_to_start():
    """Any CTA of the kernel that takes items may be cancelled by another before it starts: what the join reads is written by the
    CTA that has the item, never by one of a certain number."""
    body = _kernel_body("decode_items_kernel")
    assert body.count("header->n =") == 1 and re.search(r"if \(item == 0 && t == 0\) header->n = splits_at\[THREADS\];", body)
    assert re.findall(r"blockIdx\.x[^;]*;", body) == ["blockIdx.x) >= n_items) return;", "blockIdx.x;"]


def test_a_wait_that_runs_out_ends_alike_for_a_warp_and_a_cta():
    """Every thread has a limit of its own.  Lanes shuffle behind the wait, so a warp votes at once; the CTA votes before its next
    turn, and stays until the answer that is still under way had its time."""
    body = _kernel_body("decode_items_kernel")
    wait = body.index("mbar_wait")
    assert re.search(r"heard = __all_sync\(0xffffffffu, tc::mbar_wait\(&answered, parity, &abort_flag\)\);", body)
    vote = body.index("lost = __syncthreads_or(!heard);")
    assert wait < body.index("ring.start(") < vote < body.index("if (lost || !more) break;")
    assert re.search(r"if \(lost && t == 0\) \{\s*abort_flag = 0;\s*tc::mbar_wait\(&answered, parity \^ 1, &abort_flag\);", body[vote:])
    # between the wait and the vote a CTA's threads meet only where all of them do: at parts of an item that was begun by all
    assert body[wait:vote].count("__syncthreads") == 1
    assert body.index("if (open) {\n      unsigned char* own", wait) < body.index("__syncthreads", wait) < vote


def test_records_that_were_never_written_are_not_joined(tmp_path):
    """A CTA whose wait ran out leaves its record as the workspace had it.  Whatever 16 bytes are there, the rows that a join of
    them would write and the parts it would read lie inside; what the kernel writes itself is joined."""
    out = _run(tmp_path, r"""
#include <stdio.h>
#include <string.h>
#include "decode_join.cuh"
int main() {
  unsigned long long x = 88172645463325252ull;
  auto next = [&] { x ^= x << 13; x ^= x >> 7; x ^= x << 17; return x; };
  long long bad = 0, kept = 0, joined = 0;
  const int batches[] = {1, 3, 1 << 27}, groups[] = {1, 7, 20}, rows[] = {1, 4, 8, 16}, mosts[] = {296, 1776};
  for (int batch : batches) for (int group : groups) for (int block : rows) for (int most : mosts) {
    const int kv = 2, heads = kv * group, slots = 2 * most;
    auto check = [&](const lkv::JoinRecord& r) {
      if (!lkv::joinable(r, batch, heads, slots)) return;
      ++joined;
      const int last = group - r.head0 % group < block ? group - r.head0 % group : block;      // rows a join writes
      bad += r.b < 0 || r.b >= batch || r.head0 < 0 || (long long)r.head0 + last > heads || last < 1;
      bad += r.slot < 0 || r.parts < 1 || (long long)r.slot + r.parts > slots;
    };
    const int edges[] = {0, 1, -1, slots, slots - 1, heads - 1, heads, batch - 1, batch, 0x7fffffff, -0x7fffffff - 1};
    for (int b : edges) for (int h : edges) for (int p : edges) for (int s : edges) check({b, h, p, s});
    for (int i = 0; i < 20000; ++i) {
      lkv::JoinRecord r;
      unsigned long long w[2] = {next(), next()};
      memcpy(&r, w, sizeof(r));
      check(r);
      check({r.b % batch, r.head0 % heads, r.parts % (slots + 2), r.slot % (slots + 2)});
    }
    for (int hk = 0; hk < kv; ++hk) for (int h0 = 0; h0 < group; h0 += block)
      kept += !lkv::joinable({batch - 1, hk * group + h0, 2, slots - 2}, batch, heads, slots) || !lkv::joinable({0, h0, slots, 0}, batch, heads, slots);
    const int counts[] = {0, 5, most, most + 1, 0x7fffffff, -1, -0x7fffffff - 1};
    for (int n : counts) bad += lkv::join_count(n, most) < 0 || lkv::join_count(n, most) > most || (n >= 0 && n <= most && lkv::join_count(n, most) != n);
  }
  printf("%lld %lld %d\n", bad, kept, joined > 1000);
}
""")
    assert out == ["0", "0", "1"]
    body = _kernel_body("decode_join_kernel")
    assert "join_count(header->n, most)" in body
    assert body.index("records[i_rec]") < body.index("if (!joinable(") < body.index("rec.head0 %") < body.index("rec.parts") < body.index("rec.slot")


@pytest.mark.parametrize("source, kernels", [("lightkv_decode", 56), ("lightkv_pages", 4)])
def test_no_serving_kernel_spills(tmp_path, source, kernels):
    """Every instance that the library holds, as the compiler reports it."""
    log = subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")] + entry.NVCC_FLAGS + [
        "-Xptxas", "-v", "-cubin", "-o", str(tmp_path / "out.cubin"), os.path.join(entry.CSRC, source + ".cu")],
        check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT).stdout.decode()
    found = re.findall(r"Compiling entry function '(\w+)' for.*?(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", log, re.S)
    assert len(found) == kernels
    assert [f for f in found if f[1:] != ("0", "0", "0")] == []


# ------------------------------------------------------------------------------------------------------------ on a GPU

def _kernels(step):
    """Kernels `step` launches."""
    from bench import count_launches
    return count_launches(step)


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("width, longest", [(6, 0), (9000, 0), (9000, 200)])          # clusters; items and their join; clusters
def test_the_documented_loop_where_pages_run_out(L, captured, width, longest):
    """Requests that get no page, or are at their table's end, keep every row bit for bit and attend to what they hold; the others
    go on.  A page that comes free later serves the ones that waited."""
    import torch
    heads, kv_heads, dh, page = 8, 2, 64, 16
    rng = np.random.default_rng(5)
    # lengths; 1 and 2 need a page at once and there is one; 3 is at the end of a narrow table; 4 is no request; 0 needs its page at the third step
    start = [30, 32, 48, 6 * page, -1, 5]
    have = [-(-max(x, 0) // page) for x in start]
    n_pages = sum(have) + 3
    order, at, rows = [int(x) for x in rng.permutation(n_pages)], 0, []
    for m in have:
        rows.append(order[at:at + m] + [-1] * (width - m))
        at += m
    table, free, n_free = _i32(rows), _i32(order[at:] + [0] * at), _i32([1])
    k, v = (_random(rng, (n_pages, kv_heads, page, dh), torch.bfloat16) for _ in range(2))
    lens, status, slots = _i32(start), _i32([0]), torch.zeros(6, dtype=torch.int64, device="cuda")
    q, k_new, v_new = (torch.empty((6, h, dh), dtype=torch.bfloat16, device="cuda") for h in (heads, kv_heads, kv_heads))
    o = torch.empty_like(q)
    ws = torch.zeros(max(L.pages_workspace_bytes(6), L.decode_workspace_bytes(6, heads, kv_heads, dh)), dtype=torch.uint8, device="cuda")
    names = dict(L=L, longest=longest, lens=lens, table=table, free=free, n_free=n_free, slots=slots, status=status, ws=ws, q=q, k=k, v=v, o=o, k_new=k_new, v_new=v_new)
    body = compile(_documented_loop(), "documented loop", "exec")
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            exec(body, names)
    state = dict(seq_len_out=list(start), table=rows, free_pages=free.tolist(), n_free=1)
    waited = 0
    for step in range(6):
        if step == 3:                                       # two pages come back from elsewhere
            state["free_pages"] = list(state["free_pages"])
            state["free_pages"][:2] = order[at + 1:at + 3]
            state["n_free"] = 2
            free.copy_(_i32(state["free_pages"])), n_free.fill_(2)
        for t, h in ((q, heads), (k_new, kv_heads), (v_new, kv_heads)):
            t.copy_(_random(rng, (6, h, dh), torch.bfloat16))
        status.zero_()
        held = state["seq_len_out"]
        state = O.assign_pages(held, held, 1, state["table"], state["free_pages"], state["n_free"], page, 6, 1)
        want_k, want_v, _ = O.append_kv(_f64(k_new), _f64(v_new), _f64(k), _f64(v), state["slot_map"])
        if captured:
            graph.replay()
        else:
            exec(body, names)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(_f64(k), want_k)      # no old row has changed
        np.testing.assert_array_equal(_f64(v), want_v)
        assert lens.tolist() == state["seq_len_out"] and slots.tolist() == state["slot_map"] and int(status) == state["status"]
        for b, n in enumerate(lens.tolist()):
            if n <= 0:
                assert (o[b] == 0).all()
                continue
            waited += held[b] == n
            (kk, there), (vv, _) = (O.cache_rows(c, table[b].tolist(), n, page) for c in (want_k, want_v))
            ref, _, mass, span = O.attend(_f64(q[b]), kk, vv, there, dh ** -0.5)
            rel = 2.0 ** -22 * (dh + 4) * span + 2.0 ** -20 + 2.0 ** -16 + 2.0 ** -22 * n
            assert (np.abs(_f64(o[b]) - ref) <= 2.0 ** -8 * np.abs(ref) + rel[:, None] * mass).all(), (step, b)
    assert waited >= 4 and lens.tolist()[2] > 48             # some waited, and were served later


# one request a thread up to 256, several up to 1024, chunks of 1024 behind that; one kernel up to 1024 requests and 4096 slots
@pytest.mark.gpu
@pytest.mark.parametrize("n_slots, stride", [(4096, 0), (4097, 0), (0, 0), (2048, 2)])
@pytest.mark.parametrize("batch", [255, 256, 257, 512, 513, 1024, 1025, 2048, 2049])
def test_assign_pages_where_its_forms_meet(L, batch, n_slots, stride):
    rng = np.random.default_rng(batch + n_slots)
    for tight in (False, True):
        case = _random_pages(rng, batch, 3, 5, tight)
        want = O.assign_pages(**case, add=1, n_slots=n_slots, slot_stride=stride)
        for in_place in (None, "held"):
            got = _call_pages(L, **case, add=1, n_slots=n_slots, slot_stride=stride, in_place=in_place)
            for key in want:
                assert got[key] == want[key], (key, tight, in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 7, 0])
def test_decode_attention_new_rows_of_some_requests(L, dtype, page):
    """A slot map of any signs, in both forms, paged and contiguous, with two blocks of query heads: a request without a new row
    reads its last old one, and the cache keeps it."""
    import torch
    lens = [1, 16, 17, 33, 300, 0, 48, -1, 64, 2]
    slots = [-1, -1, 5, -7, -1, -1, 0, 3, 2 ** 62, -2 ** 62]
    c = Decode(lens, 40, 2, 64, page, dtype, new=True, width=40000 // page if page else None)
    before = c.k.clone(), c.v.clone()
    c.k_new.masked_fill_((torch.tensor(slots) < 0).cuda()[:, None, None], math.nan)          # what is not used may be anything
    where = [None if n <= 0 else (int(c.table[b, (n - 1) // page]), (n - 1) % page) if page else (b, n - 1) for b, n in enumerate(lens)]
    fresh = c.k_new, c.v_new
    c.k_new = c.v_new = None
    rows = [O.with_new_row(k, v, _f64(fresh[0][b]), _f64(fresh[1][b]), slots[b]) + (there,) for b, (k, v, there) in enumerate(c.rows())]
    for x, y in zip((c.k, c.v), fresh):
        for b, at in enumerate(where):
            if at and slots[b] >= 0:
                x[at[0], :, at[1]] = y[b]
    after = c.k.clone(), c.v.clone()
    c.k_new, c.v_new = fresh
    for hint in (0, 300, 16) if page else (0,):
        c.k.copy_(before[0]), c.v.copy_(before[1])
        c.out.fill_(math.nan), c.lse.fill_(math.nan)
        c.run(L, max_keys=hint, slot_map=torch.tensor(slots, device="cuda"))
        c.check(rows)
        for x, y in zip((c.k, c.v), after):
            assert ((x == y) | (x.isnan() & y.isnan())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [2, 14])
def test_decode_attention_infinite_logits_and_values(L, dtype, heads):
    """+inf, -inf and NaN in keys and infinite values, at the first key, the last, in several pieces and several parts of a cut
    request: out and lse as the formulas have them in 64 bits, and rows of other heads within their tolerance."""
    import torch
    lens = [40, 40, 40, 40, 3000, 3000, 3000, 40, 17, 40]
    c = Decode(lens, heads, 2, 64, 16, dtype, width=2500)
    c.q.abs_()
    inf, nan = math.inf, math.nan
    keys = [(0, 0, inf), (1, 39, inf), (2, 3, inf), (2, 20, inf), (3, 5, inf), (3, 38, nan), (4, 2999, inf), (5, 7, inf), (5, 1500, inf),
            (5, 2990, -inf), (6, 1, inf), (6, 2800, nan), (8, 16, -inf)]
    keys += [(7, j, -inf) for j in range(40) if j != 11] + [(7, 11, inf)]
    for b, j, x in keys:
        c.k[int(c.table[b, j // 16]), 0, j % 16, 9] = x
    c.v[int(c.table[9, 1]), 0, 5, 3] = inf
    c.v[int(c.table[9, 0]), 0, 7, 4] = -inf
    q, rows = _f64(c.q), list(c.rows())

    def near(out, lse, exact, n):
        ref, ref_lse, mass, span = exact
        d = 2.0 ** -23 * 68 * span
        rel = 2 * d + 2.0 ** -20 + (2.0 ** -16 if dtype == "bf16" else 0) + 2.0 ** -22 * n
        assert (np.abs(out - ref) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + rel[:, None] * mass).all()
        assert (np.abs(lse - ref_lse) <= d + 2.0 ** -20 + 2.0 ** -22 * n + 2.0 ** -22 * np.abs(ref_lse)).all()

    for hint in (0, 3000, 40, 1):
        c.out.fill_(nan), c.lse.fill_(nan)
        c.run(L, max_keys=hint)
        out, lse = _f64(c.out), _f64(c.lse)
        assert int(c.status) == 0
        for b, (k, v, _) in enumerate(rows):
            for h in range(heads // 2):                     # heads that read the first key head
                if b == 9:                                  # infinite values
                    assert not np.isfinite(out[b, h, [3, 4]]).any() and np.isfinite(np.delete(out[b, h], [3, 4])).all() and np.isfinite(lse[b, h])
                    if dtype == "fp32":
                        assert out[b, h, 3] == inf and out[b, h, 4] == -inf
                    continue
                with np.errstate(invalid="ignore"):
                    s = 0.125 * (k[0] @ q[b, h])
                if b == 8:                                  # a key without weight
                    near(out[b, h:h + 1], lse[b, h:h + 1], O.attend(q[b, h:h + 1], k[:1, :16], v[:1, :16], np.ones(16, bool), 0.125), 17)
                    continue
                assert np.isnan(out[b, h]).all(), (hint, b, h)
                assert np.isnan(lse[b, h]) if np.isnan(s).any() else lse[b, h] == inf, (hint, b, h, lse[b, h])
        half = heads // 2                                   # the other key head has nothing of it
        for b, (k, v, there) in enumerate(rows):
            near(out[b, half:], lse[b, half:], O.attend(q[b, half:], k[1:], v[1:], there, 0.125), lens[b])


def _odd(t, dims):
    """The same elements, with strides of one element more than a row where a dimension has a single one."""
    assert all(t.shape[d] == 1 for d in dims)
    return t.as_strided(t.shape, [t.shape[-1] + 1 if d in dims else s for d, s in enumerate(t.stride())], t.storage_offset())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_of_single_elements_do_not_matter(L, dtype):
    """One request, one head, one page, one row a page or one token: the stride of that dimension may be anything."""
    import torch
    c = Decode([1], 1, 1, 64, 1, dtype, new=True, spare=0)
    c.k_new, c.v_new = c.k_new.clone(), c.v_new.clone()
    assert c.k.shape == (1, 1, 1, 64)
    rows = list(c.rows())
    c.q, c.out, c.k_new, c.v_new = (_odd(t, (0, 1)) for t in (c.q, c.out, c.k_new, c.v_new))
    c.k, c.v = _odd(c.k, (0, 1, 2)), _odd(c.v, (0, 1, 2))
    c.run(L)
    c.check(rows)
    assert (c.k[0, 0, 0] == c.k_new[0, 0]).all()
    fresh = _odd(_random(np.random.default_rng(1), (1, 1, 64), c.dt), (0, 1))
    L.append_kv(fresh, fresh, c.k, c.v, torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert (c.k[0, 0, 0] == fresh[0, 0]).all() and (c.v[0, 0, 0] == fresh[0, 0]).all()
    # contiguous, one request of several rows
    c = Decode([9], 2, 1, 64, 0, dtype)
    rows = list(c.rows())
    c.q, c.out, c.k, c.v = _odd(c.q, (0,)), _odd(c.out, (0,)), _odd(c.k, (0, 1)), _odd(c.v, (0, 1))
    c.run(L)
    c.check(rows)
    with pytest.raises(L.LightKVError):                     # a stride that counts is refused as before
        L.decode_attention(torch.zeros((2, 2, 72), dtype=c.dt, device="cuda").as_strided((2, 2, 64), (145, 72, 1)), c.k.expand(2, -1, -1, -1),
                           c.v.expand(2, -1, -1, -1), _i32([1, 1]), torch.zeros((2, 2, 64), dtype=c.dt, device="cuda"), workspace=c.workspace)


@pytest.mark.gpu
def test_a_bound_of_the_keys_counts_for_contiguous_caches_too(L):
    """Caches with room for many more rows than are in use: without a bound items and their join are launched, with one a cluster.
    The bound chooses how the work is split and cuts nothing: a wrong one gives the same rows."""
    import torch
    # 6 requests and heads make 48 CTAs of 16 warps in clusters of eight: 40000 keys are 20 rounds of their warps, 64000 are 32, and items
    # are taken from rounds * (64 - 48) > 350 on
    for room, cases in ((40000, ((0, 1), (400, 1))), (64000, ((0, 2), (400, 1), (64000, 2), (70000, 2), (20, 1)))):
        c = Decode([400, 37, 0], 4, 2, 64, 0, new=True)
        k, v = (torch.full((3, 2, room, 64), math.nan, dtype=c.dt, device="cuda") for _ in range(2))
        k[:, :, :c.k.shape[2]], v[:, :, :c.v.shape[2]] = c.k, c.v
        rows = list(c.rows())
        c.k, c.v = k, v
        for bound, kernels in cases:
            c.out.fill_(math.nan), c.lse.fill_(math.nan)
            c.run(L, max_keys=bound)
            c.check(rows)
            assert _kernels(lambda: c.run(L, max_keys=bound)) == kernels, (room, bound)
    paged = Decode([400, 37, 0], 4, 2, 64, 16, width=4000)
    paged.run(L)
    assert [_kernels(lambda: paged.run(L, max_keys=bound)) for bound in (0, 400)] == [2, 1]


@pytest.mark.gpu
def test_the_smoke_run_takes_both_forms(L, monkeypatch):
    kernels, call = [], L.decode_attention

    def counted(*args, **kw):
        kernels.append(_kernels(lambda: call(*args, **kw)))
        call(*args, **kw)

    monkeypatch.setattr(L, "decode_attention", counted)
    entry._smoke_serving()
    assert kernels == [2, 1]
