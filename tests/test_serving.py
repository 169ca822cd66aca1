"""The serving calls (assign_pages, append_kv, decode_attention) against the oracle, and their refusals.

Tolerances of the attention, before any run.  u is half a step of the stored type (bf16 2^-8, fp32 2^-24) and counts once, for
the output row.  A logit is a dot product of dh fp32 terms and a scaling: it is off by at most
d = 2^-23 (dh + 4) max_j sum |q k| scale, and a weight by 2 d + 2^-21 of itself (two exponentials of 2^-22 each).  bf16 weights
are two bf16 summands, 2^-16 of themselves off.  A sum of n terms is off by 2^-23 n of the sum of their magnitudes, and a sum
over parts by as much again.  So
  |out - exact| <= u |exact| + (2 d + 2^-20 + [bf16] 2^-16 + 2^-22 n) sum_j p_j |v_j|,   |lse - exact| <= d + 2^-20 + 2^-22 n + 2^-22 |lse|.
Page numbers, lengths and slots are equal; rows that are moved are bit for bit what they were."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import __graft_entry__ as entry
from oracle import serving as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    entry.build()
    import paper_2605_00789_b200 as pkg
    return pkg


# ------------------------------------------------------------------------------------------------------ without a GPU

def test_struct_layouts_match_the_header(L, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('''#include <stdio.h>
#include <stddef.h>
#include "lightkv.h"
int main(void) {
  printf("%zu %zu %zu\\n", sizeof(lightkv_pages_args_t), offsetof(lightkv_pages_args_t, slot_map), offsetof(lightkv_pages_args_t, stream));
  printf("%zu %zu %zu\\n", sizeof(lightkv_append_args_t), offsetof(lightkv_append_args_t, k_cache), offsetof(lightkv_append_args_t, stream));
  printf("%zu %zu %zu\\n", sizeof(lightkv_decode_args_t), offsetof(lightkv_decode_args_t, block_table), offsetof(lightkv_decode_args_t, stream));
  printf("%u %u %u\\n", LIGHTKV_STATUS_COUNT, LIGHTKV_STATUS_PAGE, LIGHTKV_STATUS_NO_PAGES);
  return 0;
}
''')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    rows = [tuple(int(v) for v in line.split()) for line in subprocess.check_output([str(exe)]).decode().splitlines()]
    k = L.lightkv
    assert rows == [(C.sizeof(k._PagesArgs), k._PagesArgs.slot_map.offset, k._PagesArgs.stream.offset),
                    (C.sizeof(k._AppendArgs), k._AppendArgs.k_cache.offset, k._AppendArgs.stream.offset),
                    (C.sizeof(k._DecodeArgs), k._DecodeArgs.block_table.offset, k._DecodeArgs.stream.offset),
                    (L.STATUS_COUNT, L.STATUS_PAGE, L.STATUS_NO_PAGES)]
    assert (O.COUNT, O.PAGE, O.NO_PAGES) == rows[3]


def _pages_args(L, **kw):
    k = L.lightkv
    a = k._PagesArgs(C.sizeof(k._PagesArgs), 4, 16, 8, 64, 1)
    for i, f in enumerate(("held", "seq_len", "seq_len_out", "block_table", "free_pages", "n_free", "n_free_out", "slot_map", "slot_start")):
        setattr(a, f, 0x10000 * (i + 1))
    a.n_slots, a.workspace, a.workspace_bytes = 4, 0x1000000, L.pages_workspace_bytes(4) - 256
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("kw, code", [
    (dict(struct_size=8), -1), (dict(batch=0), -1), (dict(batch=-1), -1), (dict(page_size=0), -1), (dict(max_blocks=0), -1),
    (dict(n_pages=0), -1), (dict(add=-1), -1), (dict(n_slots=-1), -1), (dict(slot_stride=-1), -1), (dict(seq_len=None), -1),
    (dict(seq_len_out=None), -1), (dict(block_table=None), -1), (dict(free_pages=None), -1), (dict(n_free=None), -1),
    (dict(n_free_out=None), -1), (dict(workspace=None), -1), (dict(max_blocks=1 << 27), -1), (dict(slot_map=None), -1),
    (dict(n_slots=0), -1), (dict(slot_map=None, n_slots=0, slot_stride=1), -1), (dict(slot_map=0x80004), -1),
    (dict(free_pages=0x40000), -1), (dict(n_pages=2 ** 31 - 1), -2), (dict(workspace=0x1000080), -3), (dict(workspace_bytes=128), -3)])
def test_assign_pages_refuses(L, kw, code):
    assert L.library().lightkv_assign_pages(C.byref(_pages_args(L, **kw))) == code


def _append_args(L, **kw):
    k = L.lightkv
    a = k._AppendArgs(C.sizeof(k._AppendArgs), 3, 2, 64, 0, 16, 4)
    a.k_new, a.v_new, a.k_cache, a.v_cache, a.slot_map = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000
    a.new_token_stride, a.new_head_stride, a.page_stride, a.head_stride, a.row_stride = 128, 64, 2048, 1024, 64
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("kw, code", [
    (dict(struct_size=8), -1), (dict(n_tokens=-1), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=12), -1), (dict(head_dim=0), -1),
    (dict(head_dim=264, row_stride=264), -2), (dict(dtype=2), -1), (dict(page_size=0), -1), (dict(n_pages=0), -1), (dict(k_new=None), -1),
    (dict(v_cache=None), -1), (dict(slot_map=None), -1), (dict(k_new=0x1008), -1), (dict(row_stride=60), -1), (dict(head_stride=1028), -1),
    (dict(row_stride=56), -1), (dict(k_cache=0x4000), -1), (dict(k_new=0x3000), -1), (dict(n_kv_heads=4096), -2)])
def test_append_kv_refuses(L, kw, code):
    assert L.library().lightkv_append_kv(C.byref(_append_args(L, **kw))) == code


def test_append_kv_of_no_tokens_is_nothing(L):
    assert L.library().lightkv_append_kv(C.byref(_append_args(L, n_tokens=0, k_new=None, v_new=None, slot_map=None))) == 0


def _decode_args(L, **kw):
    k = L.lightkv
    a = k._DecodeArgs(C.sizeof(k._DecodeArgs), 2, 8, 2, 64, 0, 0.0, 16, 8, 32, 0)
    a.q, a.k_cache, a.v_cache, a.block_table, a.n_keys, a.out = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000
    a.q_batch_stride, a.q_head_stride, a.out_batch_stride, a.out_head_stride = 512, 64, 512, 64
    a.page_stride, a.head_stride, a.row_stride = 2048, 1024, 64
    a.workspace, a.workspace_bytes = 0x1000000, L.decode_workspace_bytes(2, 8, 2, 64) - 256
    for f, v in kw.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("kw, code", [
    (dict(struct_size=8), -1), (dict(batch=0), -1), (dict(n_q_heads=7), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=20), -1),
    (dict(head_dim=264, row_stride=264), -2), (dict(dtype=3), -1), (dict(q=None), -1), (dict(k_cache=None), -1), (dict(v_cache=None), -1),
    (dict(block_table=None), -1), (dict(n_keys=None), -1), (dict(out=None), -1), (dict(workspace=None), -1), (dict(k_new=0x7000), -1),
    (dict(page_size=-1), -1), (dict(max_blocks=0), -1), (dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(max_keys=-1), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(q=0x1008), -1), (dict(out=0x1000), -1),
    (dict(row_stride=56), -1), (dict(row_stride=68), -1), (dict(q_head_stride=68), -1), (dict(workspace=0x1000010), -3),
    (dict(workspace_bytes=16), -3), (dict(batch=1 << 27), -2), (dict(page_stride=-2048), -1), (dict(page_stride=1 << 40), -2),
    (dict(max_blocks=1 << 27, batch=1 << 9), -2), (dict(k_new=0x7000, v_new=0x8000, v_cache=0x2000), -1)])
def test_decode_attention_refuses(L, kw, code):
    assert L.library().lightkv_decode_attention(C.byref(_decode_args(L, **kw))) == code


def test_workspace_sizes(L):
    for bad in ((0, 8, 2, 64), (2, 7, 2, 64), (2, 8, 0, 64), (2, 8, 2, 60), (2, 8, 2, 264), (2, 8, 2, 64, 5)):
        with pytest.raises(L.LightKVError):
            L.decode_workspace_bytes(*bad)
    with pytest.raises(L.LightKVError):
        L.pages_workspace_bytes(-1)
    assert L.decode_workspace_bytes(256, 128, 8, 256) <= 32 << 20                # a fixed bound, whatever the lengths
    assert L.pages_workspace_bytes(1000) > L.pages_workspace_bytes(10)


def test_the_binding_refuses_tensors_of_the_host(L):
    import torch
    q, cache = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16)
    n, ws = torch.zeros((2,), dtype=torch.int32), torch.zeros((1024,), dtype=torch.uint8)
    L.lightkv._binding()
    if torch.cuda.is_available():
        with pytest.raises(ValueError, match="not on the current CUDA device"):
            L.decode_attention(q, cache, cache.clone(), n, torch.empty_like(q), workspace=ws)
    else:                                                                          # no current device to ask for
        with pytest.raises((RuntimeError, AssertionError, ValueError)):
            L.decode_attention(q, cache, cache.clone(), n, torch.empty_like(q), workspace=ws)


# kernel -> registers a thread may have for the CTAs per SM that the launches count on; none of them spills
LIMITS = {"decode_cluster_kernel<WarpBf16<2, 1>, 8, 3, 1>": 255, "decode_cluster_kernel<WarpBf16<2, 1>, 4, 3, 2>": 255,
          "decode_cluster_kernel<WarpBf16<1, 1>, 16, 3, 1>": 128, "decode_cluster_kernel<WarpBf16<1, 2>, 16, 3, 1>": 128,
          "decode_cluster_kernel<WarpBf16<2, 1>, 2, 3, 3>": 255, "decode_items_kernel<WarpBf16<2, 1>, 4, 3, 2>": 255,
          "decode_items_kernel<WarpBf16<2, 2>, 4, 3, 2>": 255, "decode_items_kernel<WarpBf16<1, 1>, 4, 6, 2>": 255}


def test_registers_and_spills(tmp_path):
    import re
    log = subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")] + entry.NVCC_FLAGS + [
        "-Xptxas", "-v", "-cubin", "-o", str(tmp_path / "out.cubin"), os.path.join(entry.CSRC, "lightkv_decode.cu")],
        check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT).stdout.decode()
    log = subprocess.run(["c++filt"], input=log.replace("'_Z", "' _Z"), check=True, capture_output=True, text=True).stdout
    log = log.replace("lkv::(anonymous namespace)::", "")
    found = {k: (int(re.search(r"Used (\d+) registers", r).group(1)), int(re.search(r"(\d+) bytes spill loads", r).group(1)))
             for k, r in re.findall(r"Compiling entry function '\s*(.*?)' for(.*?Used \d+ registers)", log, re.S)}
    for kernel, limit in LIMITS.items():
        (registers, spilled), = [v for k, v in found.items() if kernel + "(" in k]
        assert registers <= limit and spilled == 0, (kernel, registers, spilled)


def test_oracle_against_a_library_softmax():
    from scipy.special import logsumexp, softmax
    rng = np.random.default_rng(3)
    q, cache_k, cache_v = rng.standard_normal((4, 8)), rng.standard_normal((5, 2, 3, 8)), rng.standard_normal((5, 2, 3, 8))
    pages = [4, 0, 2]
    k, there = O.cache_rows(cache_k, pages, 8, 3)
    v, _ = O.cache_rows(cache_v, pages, 8, 3)
    out, lse, mass, span = O.attend(q, k, v, there, 0.3)
    for h in range(4):
        keys = np.stack([cache_k[pages[j // 3], h // 2, j % 3] for j in range(8)])
        vals = np.stack([cache_v[pages[j // 3], h // 2, j % 3] for j in range(8)])
        s = 0.3 * keys @ q[h]
        np.testing.assert_allclose(out[h], softmax(s) @ vals, rtol=1e-12)
        assert lse[h] == pytest.approx(logsumexp(s)) and (mass[h] >= np.abs(out[h]) - 1e-12).all() and span[h] >= np.abs(s).max()


def test_oracle_pages_by_hand():
    got = O.assign_pages([5, 9, 0], [2, 9, -1], 0, [[7, 8, 0], [1, 2, 3], [0, 0, 0]], [6, 5, 0, 0, 0, 0, 0, 0, 0], 2, 4, 4)
    assert got["seq_len_out"] == [2, 9, -1] and got["free_pages"][:got["n_free"]] == [6, 5, 8] and got["status"] == 0
    got = O.assign_pages([5, 4, 0], [2, 5, 3], 1, [[7, 8, 0], [1, 0, 0], [0, 0, 0]], [6, 5, 0, 0, 0, 0, 0, 0, 0], 1, 4, 8)
    # page 8 comes back, goes to request 1; request 2 gets page 6
    assert got["table"] == [[7, 8, 0], [1, 8, 0], [6, 0, 0]] and got["n_free"] == 0 and got["seq_len_out"] == [3, 6, 4]
    assert got["slot_map"] == [32, 33, 24, 25, 26, 27, -1, -1] and got["slot_start"] == [0, 0, 2, 6]
    got = O.assign_pages(None, [9, 1], 0, [[0, 0, 0], [0, 0, 0]], [6, 5, 4], 2, 4, 2, 1)
    assert got["status"] == O.NO_PAGES | O.COUNT and got["seq_len_out"] == [0, 0] and got["slot_map"] == [-1, -1] and got["n_free"] == 2


# ------------------------------------------------------------------------------------------------------------ on a GPU

def _i32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _call_pages(L, held, seq_len, add, table, free_pages, n_free, page_size, n_slots=0, slot_stride=0, in_place=None, workspace=None):
    import torch
    batch = len(seq_len)
    t = dict(seq=_i32(seq_len), table=_i32(table), free=_i32(free_pages), n_free=_i32([n_free]), status=_i32([0]))
    t["held"] = None if held is None else t["seq"] if in_place == "seq" else _i32(held)
    out = {"held": t["held"], "seq": t["seq"], None: torch.full((batch,), 77, dtype=torch.int32, device="cuda")}[in_place]
    n_out = t["n_free"] if in_place else _i32([-5])
    slots = torch.full((n_slots,), -7, dtype=torch.int64, device="cuda") if n_slots else None
    start = _i32([-7] * (batch + 1))
    ws = workspace if workspace is not None else torch.full((L.pages_workspace_bytes(batch),), 255, dtype=torch.uint8, device="cuda")
    L.assign_pages(t["seq"], t["table"], t["free"], t["n_free"], page_size=page_size, add=add, held=t["held"], seq_len_out=out,
                   n_free_out=n_out, slot_map=slots, slot_start=start, slot_stride=slot_stride, status=t["status"], workspace=ws)
    return dict(seq_len_out=out.tolist(), table=t["table"].tolist(), free_pages=t["free"].tolist(), n_free=int(n_out),
                slot_map=slots.tolist() if n_slots else [], slot_start=start.tolist(), status=int(t["status"]))


def _random_pages(rng, batch, page_size, width, tight=False, idle=0.15):
    room = width * page_size
    held = [int(rng.integers(0, room + 1)) if rng.random() > idle else int(rng.choice([0, -1, -3])) for _ in range(batch)]
    have = [-(-max(h, 0) // page_size) for h in held]
    seq = []
    for h in held:
        kind = rng.integers(0, 6)
        seq.append(-1 if rng.random() < idle else [max(h, 0), int(rng.integers(0, room + 1)), min(max(h, 0) + 1, room), max(h, 0) // 2, 0,
                                                   min(max(h, 0) + int(rng.integers(0, 3 * page_size)), room)][kind])
    n_pages = sum(have) + int(rng.integers(1, batch * width // 2 + 2))
    order = [int(v) for v in rng.permutation(n_pages)]
    table, at = [], 0
    for n in have:
        table.append(order[at:at + n] + [int(v) for v in rng.integers(-5, n_pages + 5, width - n)])
        at += n
    n_free = n_pages - at
    if tight:
        n_free = min(n_free, int(rng.integers(0, 4)))
    free = order[at:at + n_free]
    return dict(held=held, seq_len=seq, table=table, free_pages=free + [-9] * (n_pages - len(free)), n_free=n_free, page_size=page_size)


# 768 rows of requests fit on chip, 1024 are summed at once, up to 4096 slots are written by the first kernel
@pytest.mark.gpu
@pytest.mark.parametrize("batch, page_size, width, n_slots, stride, tight", [
    (1, 16, 4, 70, 0, False), (1, 1, 1, 1, 0, True), (7, 16, 9, 300, 0, False), (33, 7, 5, 33, 1, False), (64, 16, 40, 0, 0, False),
    (64, 16, 40, 4097, 0, True), (257, 1, 6, 700, 2, False), (768, 4, 3, 4096, 0, True), (769, 4, 3, 900, 1, False),
    (1024, 3, 4, 5000, 0, True), (1025, 16, 3, 4100, 4, True), (2500, 2, 3, 2500, 1, True), (300, 64, 20, 100000, 0, False)])
def test_assign_pages(L, batch, page_size, width, n_slots, stride, tight):
    rng = np.random.default_rng(batch * 31 + width)
    for add in (0, 1):
        case = _random_pages(rng, batch, page_size, width, tight)
        want = O.assign_pages(**case, add=add, n_slots=n_slots, slot_stride=stride)
        for in_place in (None, "held"):
            got = _call_pages(L, **case, add=add, n_slots=n_slots, slot_stride=stride, in_place=in_place)
            for key in want:
                assert got[key] == want[key], (key, add, in_place)


@pytest.mark.gpu
def test_assign_pages_one_array_of_lengths_for_all_three(L):
    # a decoding step in place: held, wanted and resulting lengths are one array, some places are without a request
    rng = np.random.default_rng(8)
    lens = [int(v) for v in rng.integers(0, 40, 50)]
    lens[3] = lens[17] = -1
    lens[5], lens[6], lens[7] = 0, 15, 16
    have = [-(-max(v, 0) // 16) for v in lens]
    order, at, table = [int(v) for v in rng.permutation(200)], 0, []
    for n in have:
        table.append(order[at:at + n] + [0] * (4 - n))
        at += n
    case = dict(seq_len=lens, table=table, free_pages=order[at:] + [0] * at, n_free=200 - at, page_size=16, add=1, n_slots=50, slot_stride=1)
    want = O.assign_pages(held=lens, **case)
    got = _call_pages(L, held=lens, in_place="seq", **case)
    assert got == want and got["seq_len_out"][3] == -1 and got["seq_len_out"][5] == 1


@pytest.mark.gpu
@pytest.mark.parametrize("change, bit", [
    (dict(n_free=-3), O.COUNT), (dict(n_free=10 ** 6), O.COUNT), (dict(held=[1000, 3, 0]), O.COUNT), (dict(seq_len=[0, 2 ** 31 - 1, 4]), O.COUNT),
    (dict(free_pages=[99, -4, 8] + [0] * 9, n_free=3, seq_len=[9, 9, 9]), O.PAGE),
    (dict(seq_len=[40, 3, 4]), O.NO_PAGES), (dict(n_free=0, seq_len=[20, 3, 4]), O.NO_PAGES)])
def test_assign_pages_conditions_only_the_device_sees(L, change, bit):
    case = dict(held=[20, 3, 0], seq_len=[5, 6, 7], add=1, table=[[0, 1, 2, 3, 4, 0, 0, 0, 0, 0, 0, 0], [5] + [0] * 11, [0] * 12],
                free_pages=[6, 7, 8, 9] + [0] * 8, n_free=4, page_size=4, n_slots=40)
    case.update(change)
    if "held" in change:                                    # the table is full then
        case["table"] = [list(range(12)), [5] + [0] * 11, [0] * 12]
        case["seq_len"] = [48, 6, 7]
        case["add"] = 0
    want = O.assign_pages(**case)
    got = _call_pages(L, **case)
    assert got == want and got["status"] & bit


def _random(rng, shape, torch_dtype):
    import torch
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda").to(torch_dtype)


def _f64(t):
    return t.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens, heads, dh, page, dtype, layout", [
    (1, 1, 8, 1, "bf16", "head"), (5, 3, 72, 16, "bf16", "token"), (700, 8, 128, 16, "bf16", "head"), (3000, 2, 64, 7, "bf16", "token"),
    (33, 40, 256, 32, "fp32", "head"), (64, 1, 8, 16, "fp32", "token"), (2049, 1, 8, 5, "bf16", "head")])
def test_append_kv(L, tokens, heads, dh, page, dtype, layout):
    import torch
    rng = np.random.default_rng(tokens + dh)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_pages = tokens // page + 3
    shape = (n_pages, heads, page, dh) if layout == "head" else (n_pages, page, heads, dh)
    k_cache, v_cache = (_random(rng, shape, dt) for _ in range(2))
    if layout == "token":
        k_cache, v_cache = k_cache.permute(0, 2, 1, 3), v_cache.permute(0, 2, 1, 3)
    # new rows as slices of a wider projection: [T, 2 heads + 1, dh]
    k_new, v_new = (_random(rng, (tokens, 2 * heads + 1, dh), dt)[:, 1:heads + 1] for _ in range(2))
    slots = rng.permutation(n_pages * page)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.2] = -1
    if tokens > 4:
        slots[2], slots[3] = n_pages * page, 2 ** 40
    want_k, want_v, want = O.append_kv(_f64(k_new), _f64(v_new), _f64(k_cache), _f64(v_cache), slots)
    status = _i32([0])
    L.append_kv(k_new, v_new, k_cache, v_cache, torch.from_numpy(slots).cuda(), status=status)
    np.testing.assert_array_equal(_f64(k_cache), want_k)
    np.testing.assert_array_equal(_f64(v_cache), want_v)
    assert int(status) == want


@pytest.mark.gpu
def test_append_kv_to_a_contiguous_cache(L):
    import torch
    rng = np.random.default_rng(5)
    k_cache, v_cache = (_random(rng, (3, 2, 50, 64), torch.bfloat16) for _ in range(2))
    k_new, v_new = (_random(rng, (4, 2, 64), torch.bfloat16) for _ in range(2))
    slots = torch.tensor([0 * 50 + 7, 1 * 50 + 49, 2 * 50 + 0, 1 * 50 + 3], device="cuda")
    want_k, want_v, _ = O.append_kv(_f64(k_new), _f64(v_new), _f64(k_cache), _f64(v_cache), slots.tolist())
    L.append_kv(k_new, v_new, k_cache, v_cache, slots)
    np.testing.assert_array_equal(_f64(k_cache), want_k)
    np.testing.assert_array_equal(_f64(v_cache), want_v)


class Decode:
    """Inputs of a decode call, its run and its check."""

    def __init__(self, lens, heads, kv_heads, dh, page=16, dtype="bf16", layout="head", new=False, seed=0, width=None, spare=2, scale=None,
                 gain=2.0):
        import torch
        rng = np.random.default_rng(seed + 1000 * dh + heads)
        self.lens, self.page, self.scale = list(lens), page, scale
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        batch = len(lens)
        blocks = [-(-max(n, 0) // page) if page else 0 for n in lens]
        self.table = None
        if page:
            width = width or max(max(blocks), 1)
            n_pages = sum(blocks) + spare
            order = [int(v) for v in rng.permutation(n_pages)]
            rows, at = [], 0
            for n in blocks:
                rows.append(order[at:at + n] + [-1] * (width - n))
                at += n
            self.table = _i32(rows)
            shape = (n_pages, kv_heads, page, dh)
        else:
            shape = (batch, kv_heads, max(max(lens), 1) + 3, dh)
        if layout == "token":
            shape = (shape[0], shape[2], shape[1], shape[3])
        self.k, self.v = (_random(rng, shape, self.dt) for _ in range(2))
        if layout == "token":
            self.k, self.v = self.k.permute(0, 2, 1, 3), self.v.permute(0, 2, 1, 3)
        # what no request holds is not a number
        held = np.zeros((shape[0], self.k.shape[2]), bool)
        for b, n in enumerate(lens):
            for j in range(max(n, 0)):
                held[(rows[b][j // page], j % page) if page else (b, j)] = True
        dead = torch.from_numpy(~held).cuda()[:, None, :, None]
        for c in (self.k, self.v):
            c.masked_fill_(dead, math.nan)
        self.q = _random(rng, (batch, heads, dh), self.dt) * gain
        self.k_new = self.v_new = None
        if new:
            self.k_new, self.v_new = (_random(rng, (batch, 2 * kv_heads, dh), self.dt)[:, :kv_heads] for _ in range(2))
        self.n_keys = _i32(self.lens)
        self.out = torch.full((batch, heads, dh), math.nan, dtype=self.dt, device="cuda")
        self.lse = torch.full((batch, heads), math.nan, device="cuda")
        self.status = _i32([0])
        self.workspace = None

    def run(self, L, **kw):
        import torch
        if self.workspace is None:
            self.workspace = torch.full((L.decode_workspace_bytes(self.q.shape[0], self.q.shape[1], self.k.shape[1], self.q.shape[2],
                                                                  L.BF16 if self.dt == torch.bfloat16 else L.FP32),), 255, dtype=torch.uint8, device="cuda")
        args = dict(block_table=self.table, lse=self.lse, k_new=self.k_new, v_new=self.v_new, workspace=self.workspace, status=self.status)
        if self.scale is not None:
            args["scale"] = self.scale
        args.update(kw)
        L.decode_attention(self.q, self.k, self.v, self.n_keys, self.out, **args)

    def rows(self, lens=None):
        """Every request's K and V rows with the new row in place, as the oracle takes them."""
        k, v = _f64(self.k), _f64(self.v)
        table = None if self.table is None else self.table.tolist()
        for b, n in enumerate(self.lens if lens is None else lens):
            n = max(n, 0)
            if self.page:
                n = min(n, len(table[b]) * self.page)
                kk, there = O.cache_rows(k, table[b], n, self.page)
                vv, _ = O.cache_rows(v, table[b], n, self.page)
            else:
                n = min(n, k.shape[2])
                kk, vv, there = k[b][:, :n], v[b][:, :n], np.ones(n, bool)
            if n and self.k_new is not None:
                kk[:, n - 1], vv[:, n - 1] = _f64(self.k_new[b]), _f64(self.v_new[b])
            yield kk, vv, there

    def check(self, rows=None, status=0):
        import torch
        q, out, lse = _f64(self.q), _f64(self.out), _f64(self.lse)
        dh = q.shape[2]
        scale = self.scale if self.scale is not None else dh ** -0.5
        bf16 = self.dt == torch.bfloat16
        u = 2.0 ** -8 if bf16 else 2.0 ** -24
        for b, (k, v, there) in enumerate(self.rows() if rows is None else rows):
            ref, ref_lse, mass, span = O.attend(q[b], k, v, there, scale)
            n = int(there.sum())
            if n == 0:
                assert (out[b] == 0).all() and (lse[b] == -math.inf).all(), b
                continue
            d = 2.0 ** -23 * (dh + 4) * span
            rel = 2 * d + 2.0 ** -20 + (2.0 ** -16 if bf16 else 0) + 2.0 ** -22 * n
            off = np.abs(out[b] - ref) - u * np.abs(ref) - rel[:, None] * mass
            assert (off <= 0).all(), (b, n, float(off.max()), np.argwhere(~(off <= 0))[:4].tolist())
            off = np.abs(lse[b] - ref_lse) - (d + 2.0 ** -20 + 2.0 ** -22 * n + 2.0 ** -22 * np.abs(ref_lse))
            assert (off <= 0).all(), (b, n, "lse", float(off.max()))
        assert int(self.status) == status


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, -1, 255, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("heads, kv_heads, dh, page, dtype, layout, new", [
    (8, 2, 128, 16, "bf16", "head", False), (8, 2, 128, 16, "bf16", "head", True), (4, 4, 64, 16, "bf16", "token", True),
    (7, 1, 128, 7, "bf16", "head", True), (32, 2, 128, 32, "bf16", "token", False), (9, 1, 64, 1, "bf16", "head", True),
    (20, 1, 96, 24, "bf16", "head", False), (6, 3, 80, 16, "bf16", "token", True), (4, 2, 256, 64, "bf16", "head", True),
    (12, 1, 256, 16, "bf16", "head", False), (3, 3, 8, 16, "bf16", "head", True), (2, 1, 72, 256, "bf16", "token", True),
    (5, 1, 200, 5, "bf16", "head", False), (40, 1, 32, 16, "bf16", "head", True),
    (4, 4, 128, 16, "fp32", "head", False), (8, 2, 128, 16, "fp32", "token", True), (7, 1, 64, 7, "fp32", "head", True),
    (9, 1, 96, 16, "fp32", "head", False), (2, 2, 256, 16, "fp32", "token", True), (12, 2, 200, 32, "fp32", "head", True),
    (3, 3, 8, 1, "fp32", "head", True)])
def test_decode_attention_at_the_edges(L, heads, kv_heads, dh, page, dtype, layout, new):
    # a table of 40000 keys a request: cut into items, joined by a second kernel; with the longest request announced: in clusters
    c = Decode(EDGES, heads, kv_heads, dh, page, dtype, layout, new, width=40000 // page)
    rows = list(c.rows())
    before = (c.k.clone(), c.v.clone())
    for hint in (0, 300, 16, 1):
        c.out.fill_(math.nan)
        c.lse.fill_(math.nan)
        c.run(L, max_keys=hint)
        c.check(rows)
    # only the new rows have changed
    for cache, old, fresh in ((c.k, before[0], c.k_new), (c.v, before[1], c.v_new)):
        if new:
            for b, n in enumerate(EDGES):
                if n > 0:
                    page_no = int(c.table[b, (n - 1) // page])
                    assert (cache[page_no, :, (n - 1) % page] == fresh[b]).all()
                    old[page_no, :, (n - 1) % page] = fresh[b]
        assert ((cache == old) | (cache.isnan() & old.isnan())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("batch, heads, kv_heads, longest", [
    (1, 8, 8, 700), (1, 4, 1, 5000), (1, 1, 1, 40000), (3, 7, 7, 900), (2, 28, 4, 9000), (37, 8, 4, 400), (150, 4, 2, 260), (300, 2, 2, 90),
    (64, 16, 8, 1500), (5, 40, 40, 333), (1, 16, 1, 20000), (128, 8, 8, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_attention_batches(L, batch, heads, kv_heads, longest, dtype):
    if dtype == "fp32" and batch * longest * kv_heads > 60000:
        longest = max(1, 60000 // (batch * kv_heads))
    seen = {}
    rng = np.random.default_rng(batch)
    lens = [int(v) for v in np.exp(rng.uniform(0, math.log(longest), batch))]
    lens[-1] = longest
    c = Decode(lens, heads, kv_heads, 64 if longest < 9000 else 128, 16, dtype, new=batch % 2 == 0, width=4000)
    rows = list(c.rows())
    for hint in (0, longest, 0, longest):                   # the hint chooses how the work is split, no more
        c.out.fill_(math.nan)
        c.lse.fill_(math.nan)
        c.run(L, max_keys=hint)
        c.check(rows)
        first = seen.setdefault(hint, (c.out.clone(), c.lse.clone()))
        assert (c.out == first[0]).all() and (c.lse == first[1]).all()   # bit for bit, run after run


@pytest.mark.gpu
@pytest.mark.parametrize("heads, kv_heads, dh, page, dtype, new", [
    (4, 2, 128, 16, "bf16", True), (16, 1, 128, 7, "bf16", False), (5, 5, 64, 16, "bf16", True), (12, 1, 64, 1, "bf16", False), (9, 1, 256, 16, "bf16", True),
    (3, 1, 96, 32, "bf16", False), (1, 1, 256, 24, "bf16", True), (2, 2, 128, 16, "fp32", True), (8, 1, 64, 7, "fp32", False), (4, 1, 256, 16, "fp32", True)])
def test_decode_attention_many_short_requests(L, heads, kv_heads, dh, page, dtype, new):
    """More (request, head) pairs than SMs, in CTAs of two warps (up to 256 keys, or 512), of four, and of more."""
    rng = np.random.default_rng(dh)
    for longest in (60, 256, 500):
        lens = [int(v) for v in rng.integers(0, longest + 1, 470 // kv_heads)]
        lens[0], lens[1], lens[2] = longest, 1, -5
        c = Decode(lens, heads, kv_heads, dh, page, dtype, new=new)
        rows = list(c.rows())
        for hint in (0, 1100):
            c.out.fill_(math.nan)
            c.lse.fill_(math.nan)
            c.run(L, max_keys=hint)
            c.check(rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_attention_contiguous_caches(L, dtype):
    for layout in ("head", "token"):
        c = Decode([5, 0, 77, 130, 1], 8, 4, 128, 0, dtype, layout, new=True)
        rows = list(c.rows())
        c.run(L)
        c.check(rows)
        c.n_keys.copy_(_i32([5, 0, 77, 1000, 1]))           # more than a request has rows: cut, and said so
        lens = [5, 0, 77, c.k.shape[2], 1]
        c.k[3], c.v[3] = 0.5, 0.25
        rows = list(c.rows(lens))
        c.run(L)
        c.check(rows, status=O.COUNT)


@pytest.mark.gpu
def test_decode_attention_strided_views(L):
    """q and out inside wider tensors, caches as halves of one pool, lse transposed, scale given."""
    import torch
    c = Decode([3, 50, 200], 8, 4, 64, 16, scale=0.3)
    pool = torch.full((c.k.shape[0], 2, c.k.shape[2], 4, 2, 64), math.nan, dtype=c.dt, device="cuda")      # [page, K/V, row, head, spare, dh]
    pool[:, 0, :, :, 0], pool[:, 1, :, :, 0] = c.k.transpose(1, 2), c.v.transpose(1, 2)
    k, v = pool[:, 0, :, :, 0].transpose(1, 2), pool[:, 1, :, :, 0].transpose(1, 2)
    wide = torch.full((3, 20, 64), math.nan, dtype=c.dt, device="cuda")
    wide[:, 4:12] = c.q
    out = torch.full((8, 3, 64), math.nan, dtype=c.dt, device="cuda")
    lse = torch.full((8, 3), math.nan, device="cuda")
    ws = torch.empty((L.decode_workspace_bytes(3, 8, 4, 64),), dtype=torch.uint8, device="cuda")
    L.decode_attention(wide[:, 4:12], k, v, c.n_keys, out.transpose(0, 1), block_table=c.table, lse=lse.t(), scale=0.3, workspace=ws)
    c.out, c.lse = out.transpose(0, 1), lse.t()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_attention_bad_pages_are_left_out(L, dtype):
    import torch
    c = Decode([100, 33, 20, 64], 4, 2, 64, 16, dtype, new=True, spare=5)
    c.table[0, 2], c.table[0, 5], c.table[1, 0], c.table[3, 3] = -1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31
    c.table[2, :] = 10 ** 6                                 # nothing is left of request 2
    rows = list(c.rows())
    before = c.k.clone()
    c.run(L)
    c.check(rows, status=O.PAGE)
    c.status.zero_()
    assert (c.out[2] == 0).all()
    # request 3's new row had a bad page: it is left out and written nowhere
    n_changed = int((~((c.k == before) | (c.k.isnan() & before.isnan()))).any(dim=3).any(dim=1).sum())
    assert n_changed <= 2
    c.table[:, :] = -1
    c.run(L)
    assert (c.out == 0).all() and (c.lse == -math.inf).all() and int(c.status) == O.PAGE


@pytest.mark.gpu
def test_decode_attention_too_many_keys_for_the_table(L):
    c = Decode([40, 40], 4, 2, 64, 16, width=3)
    c.table[0, 2], c.table[1, 2] = c.table[0, 0], c.table[1, 1]
    c.k.nan_to_num_(0.1), c.v.nan_to_num_(0.1)
    c.n_keys.copy_(_i32([1000, 2 ** 31 - 1]))
    c.run(L)
    c.check(list(c.rows([48, 48])), status=O.COUNT)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_attention_extreme_logits(L, dtype):
    """Logits that climb by more than the range of fp32 along a request, that are all alike, and that leave one key."""
    import torch
    c = Decode([500, 500, 500, 40], 2, 1, 64, 16, dtype)
    q = torch.zeros_like(c.q)
    q[:, :, 0] = 8.0
    c.q = q
    ramp = torch.linspace(-300, 300, 500)
    for b in range(4):
        n = c.lens[b]
        for j in range(n):
            p, i = int(c.table[b, j // 16]), j % 16
            c.k[p, 0, i] = 0
            c.k[p, 0, i, 0] = float(ramp[j]) if b == 0 else float(ramp[499 - j]) if b == 1 else 0.0 if b == 2 else (400.0 if j == 23 else -400.0)
    c.run(L)
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_attention_infinities_and_nan(L, dtype):
    """-inf in all logits: an empty row.  NaN or +inf in a key or value: NaN where the formula has it, other heads untouched."""
    import torch
    c = Decode([40, 40, 40, 40], 2, 2, 64, 16, dtype)
    c.q.fill_(1.0)
    page, row = int(c.table[0, 1]), 4
    for j in range(40):                                     # request 3: every logit of head 0 is -inf
        c.k[int(c.table[3, j // 16]), 0, j % 16] = -math.inf
    c.k[page, 0, row, 3] = math.nan                         # request 0, head 0
    c.v[int(c.table[1, 0]), 1, 2, 5] = math.nan             # request 1, head 1, channel 5
    c.k[int(c.table[2, 2]), 1, 7, 0] = -math.inf            # request 2, head 1: one key without weight
    c.run(L)
    out, lse = c.out.float(), c.lse
    assert out[0, 0].isnan().all() and out[0, 1].isfinite().all() and out[1, 1, 5].isnan()
    assert out[1, 1].isnan().sum() == 1 and out[1, 0].isfinite().all() and out[2].isfinite().all()
    assert (out[3, 0] == 0).all() and lse[3, 0] == -math.inf and out[3, 1].isfinite().all()
    k, v, there = list(c.rows())[2]
    ref, ref_lse, mass, span = O.attend(_f64(c.q)[2], np.where(np.isfinite(k), k, -1e30), v, there, 0.125)
    assert np.abs(_f64(c.out)[2] - ref).max() < 2.0 ** -6 * np.abs(v).max()


@pytest.mark.gpu
@pytest.mark.parametrize("page, dtype", [(16, "bf16"), (24, "bf16"), (24, "fp32")])
def test_decode_attention_offsets_past_32_bits(L, page, dtype):
    """Pages more than 2^32 bytes (and 2^31 elements) behind the pool's start, odd token counts, in both forms."""
    import torch
    c = Decode([100, 37], 4, 2, 128, page, dtype, new=True, width=2000)
    far = 600000 if dtype == "bf16" else 400000            # pages of 8, 12, 24 KB: 4.9 to 9.8 GB
    k, v = (torch.empty((far + 16, 2, page, 128), dtype=c.dt, device="cuda") for _ in range(2))
    n = c.k.shape[0]
    k[far:far + n], v[far:far + n] = c.k, c.v
    rows = list(c.rows())
    table = torch.where(c.table >= 0, c.table + far, c.table)
    for hint in (0, 100):
        c.out.fill_(math.nan)
        L.decode_attention(c.q, k, v, c.n_keys, c.out, block_table=table, lse=c.lse, k_new=c.k_new, v_new=c.v_new, status=c.status, max_keys=hint,
                           workspace=torch.empty((L.decode_workspace_bytes(2, 4, 2, 128, L.BF16 if dtype == "bf16" else L.FP32),), dtype=torch.uint8, device="cuda"))
        c.check(rows)
    for b, last in ((0, 99), (1, 36)):
        assert (k[int(table[b, last // page]), :, last % page] == c.k_new[b]).all()
    slots = torch.tensor([(far + 3) * page + 5, (far + 9) * page], device="cuda")
    L.append_kv(c.k_new, c.v_new, k, v, slots)
    assert (k[far + 3, :, 5] == c.k_new[0]).all() and (v[far + 9, :, 0] == c.v_new[1]).all()


@pytest.mark.gpu
def test_decode_attention_streams_graphs_and_a_shared_workspace(L):
    """Another stream; a captured call replayed with other lengths; two captured calls with one workspace, replayed in turn."""
    import torch
    a, b = Decode([700, 3, 90], 8, 2, 128, 16), Decode([33, 1500, 64, 2], 8, 2, 128, 16, seed=4)
    ws = torch.full((max(L.decode_workspace_bytes(n, 8, 2, 128) for n in (3, 4)),), 255, dtype=torch.uint8, device="cuda")
    a.workspace = b.workspace = ws
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a.run(L, stream=side)
    side.synchronize()
    a.check()
    graphs = []
    for c in (a, b):
        c.out.fill_(math.nan)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(L)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    a.check()
    b.check()
    lens = [1, 0, 89]
    a.n_keys.copy_(_i32(lens))
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    a.check(list(a.rows(lens)))
    b.check()


@pytest.mark.gpu
def test_decode_attention_two_streams_at_once(L):
    """Calls that overlap on the GPU, each with its own workspace, in both forms."""
    import torch
    cs = [Decode([900, 40, 7, 2000], 8, 4, 64, 16, width=3000, seed=s) for s in range(4)]
    rows = [list(c.rows()) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    cs[0].run(L), cs[0].run(L, max_keys=2000)
    for c in cs[1:]:
        c.workspace = torch.full_like(cs[0].workspace, 255)
    torch.cuda.synchronize()
    for hint in (0, 2000):
        for c in cs:
            c.out.fill_(math.nan)
        torch.cuda.synchronize()
        for _ in range(20):
            for c, s in zip(cs, streams):
                c.run(L, stream=s, max_keys=hint)
        torch.cuda.synchronize()
        for c, r in zip(cs, rows):
            c.check(r)


@pytest.mark.gpu
def test_assign_pages_captured_steps_two_at_once(L):
    """A captured step replayed on two streams with states of their own; lengths wanted without any held, in place."""
    import torch
    rng = np.random.default_rng(17)
    states = []
    for k in range(2):
        lens = [int(v) for v in rng.integers(0, 60, 40)]
        want = O.assign_pages(None, lens, 0, [[0] * 8 for _ in lens], list(rng.permutation(400)), 400, 16)
        t = dict(seq=_i32(lens), table=_i32([[0] * 8 for _ in lens]), free=torch.zeros(400, dtype=torch.int32, device="cuda"), n=_i32([400]))
        order = [int(v) for v in rng.permutation(400)]
        t["free"].copy_(_i32(order))
        ws = torch.full((L.pages_workspace_bytes(40),), 255, dtype=torch.uint8, device="cuda")
        L.assign_pages(t["seq"], t["table"], t["free"], t["n"], page_size=16, workspace=ws)          # lengths in place of those wanted
        want = O.assign_pages(None, lens, 0, [[0] * 8 for _ in lens], order, 400, 16)
        assert t["seq"].tolist() == want["seq_len_out"] and t["table"].tolist() == want["table"] and int(t["n"]) == want["n_free"]
        slots = torch.zeros(40, dtype=torch.int64, device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            L.assign_pages(t["seq"], t["table"], t["free"], t["n"], page_size=16, add=1, held=t["seq"], slot_map=slots, slot_stride=1, workspace=ws)
        states.append((t, want, slots, stream, graph))
    for _ in range(20):
        for t, want, slots, stream, graph in states:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for t, want, slots, stream, graph in states:
        for _ in range(20):
            want = O.assign_pages(want["seq_len_out"], want["seq_len_out"], 1, want["table"], want["free_pages"], want["n_free"], 16, 40, 1)
        assert t["seq"].tolist() == want["seq_len_out"] and t["table"].tolist() == want["table"] and int(t["n"]) == want["n_free"]
        assert slots.tolist() == want["slot_map"]


@pytest.mark.gpu
def test_the_binding_checks_tensors(L):
    import torch
    c = Decode([20, 20], 4, 2, 64, 16)
    c.run(L)
    ok = dict(block_table=c.table, workspace=c.workspace)
    call = lambda q=c.q, k=c.k, v=c.v, n=c.n_keys, out=c.out, **kw: L.decode_attention(q, k, v, n, out, **{**ok, **kw})  # noqa: E731
    call()
    for err, kw in [
            (TypeError, dict(n=c.n_keys.long())), (TypeError, dict(q=c.q.half())), (TypeError, dict(k=c.k.float())), (TypeError, dict(out=c.out.float())),
            (ValueError, dict(q=c.q[:, :, :32])), (ValueError, dict(n=c.n_keys[:1])), (ValueError, dict(out=c.out[:1])), (ValueError, dict(q=c.q[0])),
            (ValueError, dict(k=c.k[:1])), (ValueError, dict(n=c.n_keys.cpu())), (ValueError, dict(block_table=c.table.cpu())),
            (ValueError, dict(block_table=c.table[:1])), (TypeError, dict(block_table=c.table.long())), (ValueError, dict(lse=c.lse[:1])),
            (TypeError, dict(lse=c.lse.half())), (ValueError, dict(k_new=c.q[:, :2])), (ValueError, dict(k_new=c.q, v_new=c.q)),
            (TypeError, dict(status=torch.zeros(1, device="cuda"))), (ValueError, dict(q=c.q.transpose(1, 2).contiguous().transpose(1, 2))),
            (ValueError, dict(v=c.v.transpose(1, 2).contiguous().transpose(1, 2))), (TypeError, dict(nonsense=1)), (L.LightKVError, dict(workspace=c.workspace[:64])),
            (L.LightKVError, dict(out=c.q)), (ValueError, dict(block_table=None))]:
        with pytest.raises(err):
            call(**kw)
    with pytest.raises(TypeError):
        L.decode_attention(c.q, c.k, c.v, c.n_keys, c.out)
    slots = torch.zeros((2,), dtype=torch.int64, device="cuda")
    new = c.q[:, :2].contiguous()
    for err, kw in [(TypeError, dict(slot_map=slots.int())), (ValueError, dict(slot_map=slots[:1])), (ValueError, dict(k_new=new[:, :1])),
                    (TypeError, dict(k_new=new.float())), (ValueError, dict(v_new=new[:1])), (L.LightKVError, dict(v_cache=c.k))]:
        with pytest.raises(err):
            L.append_kv(**{**dict(k_new=new, v_new=new, k_cache=c.k, v_cache=c.v, slot_map=slots), **kw})
    ws = torch.zeros((L.pages_workspace_bytes(2),), dtype=torch.uint8, device="cuda")
    free, n_free = _i32(list(range(c.k.shape[0]))), _i32([2])
    for err, kw in [(TypeError, dict(seq_len=c.n_keys.long())), (ValueError, dict(block_table=c.table[:1])), (ValueError, dict(held=c.n_keys[:1])),
                    (ValueError, dict(n_free=free)), (TypeError, dict(slot_map=free)), (ValueError, dict(slot_start=free[:2])),
                    (ValueError, dict(block_table=c.table.t().contiguous().t())), (L.LightKVError, dict(add=-1)), (L.LightKVError, dict(workspace=ws[:64])),
                    (L.LightKVError, dict(page_size=0)), (TypeError, dict(page_size=None))]:
        with pytest.raises(err):
            L.assign_pages(**{**dict(seq_len=c.n_keys, block_table=c.table, free_pages=free, n_free=n_free, page_size=16, workspace=ws), **kw})


@pytest.mark.gpu
def test_a_serving_run_behind_the_compression(L):
    """Prefill rows are appended, the compression shrinks the pages in place, what became free goes to a new request, and all
    decode together, the steps captured in one graph: against the oracle, token by token."""
    import torch
    rng = np.random.default_rng(11)
    page, kv_heads, heads, dh, batch, text = 4, 2, 4, 64, 3, 5
    side = 8
    n_grid, n_pages, width = side * side, 64, 24
    plan = L.Plan(batch=2, hidden=64, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=dh, n_layers=4, tiles=[(side, side)], layers=[2],
                  windows=[2], keep=[0.5], max_text=text, xi_mode=L.XI_UNIFORM)
    i32 = dict(dtype=torch.int32, device="cuda")
    k, v = (torch.full((n_pages, kv_heads, page, dh), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, free, n_free = torch.full((batch, width), -1, **i32), torch.randperm(n_pages).to(**i32), _i32([n_pages])
    lens, status = _i32([-1] * batch), _i32([0])
    ws = torch.zeros((max(L.pages_workspace_bytes(batch), L.decode_workspace_bytes(batch, heads, kv_heads, dh)),), dtype=torch.uint8, device="cuda")
    model = [np.zeros((kv_heads, 0, dh)), np.zeros((kv_heads, 0, dh))]
    hold = [[model[0].copy(), model[1].copy()] for _ in range(batch)]          # what every request holds, in float64

    def admit(new_lens):
        """New lengths for places of the batch (None: unchanged) and their rows."""
        want = [int(x) if n is None else n for n, x in zip(new_lens, lens.tolist())]
        fresh = [0 if n is None else n for n in new_lens]
        slots = torch.zeros((sum(fresh) + 2,), dtype=torch.int64, device="cuda")
        L.assign_pages(_i32(want), table, free, n_free, page_size=page, held=lens, slot_map=slots, status=status, workspace=ws)
        kn, vn = (_random(rng, (sum(fresh) + 2, kv_heads, dh), torch.bfloat16) for _ in range(2))
        L.append_kv(kn, vn, k, v, slots, status=status)
        at = 0
        for b, n in enumerate(fresh):
            if n:
                hold[b] = [np.moveaxis(_f64(x[at:at + n]), 1, 0) for x in (kn, vn)]
                at += n

    admit([text + n_grid, text + n_grid, None])
    assert int(status) == 0 and lens.tolist() == [69, 69, -1] and int(n_free) == n_pages - 36
    hidden = _random(rng, (2, text + n_grid, 64), torch.bfloat16)
    out = L.StageBuffers(plan, 0, text + plan.stage_info(0).cap_out)
    L.compress_layer(plan, 0, hidden, out, vis_begin=text)
    pages = table[:2].contiguous()
    L.compact_kv(plan, 0, out, k, v, k, v, vis_begin=text, page_size=page, src_block_table=pages, dst_block_table=pages)
    counts = torch.cat([out.n_vis_out, _i32([-1])])
    for b in range(2):                                     # the oracle's view: rows merged by the map
        n, off, src, wt = int(out.n_vis_out[b]), out.grp_off[b].tolist(), out.grp_src[b].tolist(), _f64(out.weight[b])
        for i in range(2):
            rows = hold[b][i]
            merged = [np.einsum("g,hgd->hd", wt[src[off[o]:off[o + 1]]], rows[:, [text + s for s in src[off[o]:off[o + 1]]]]) for o in range(n)]
            hold[b][i] = np.concatenate([rows[:, :text], np.stack(merged, 1)], 1)
    L.assign_pages(counts, table, free, n_free, page_size=page, add=text, held=lens, status=status, workspace=ws)
    assert lens.tolist() == [37, 37, -1] and int(n_free) == n_pages - 20 and int(status) == 0
    for b in range(2):                                      # merged rows were rounded to bf16: take them from the cache
        for i, cache in enumerate((k, v)):
            got, _ = O.cache_rows(_f64(cache), table[b].tolist(), 37, page)
            assert np.abs(got - hold[b][i]).max() <= 2.0 ** -8 * np.abs(hold[b][i]).max() + 1e-4
            hold[b][i] = got
    admit([None, None, 41])                                 # the third request takes what became free
    assert lens.tolist() == [37, 37, 41] and int(n_free) == n_pages - 31

    steps = 6
    qs, kns, vns = (_random(rng, (steps, batch, h, dh), torch.bfloat16) for h in (heads, kv_heads, kv_heads))
    q, kn, vn = (torch.empty_like(x[0]) for x in (qs, kns, vns))
    o, lse = torch.empty_like(q), torch.empty((batch, heads), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.assign_pages(lens, table, free, n_free, page_size=page, add=1, held=lens, status=status, workspace=ws)
        L.decode_attention(q, k, v, lens, o, block_table=table, lse=lse, k_new=kn, v_new=vn, status=status, workspace=ws)
    for s in range(steps):
        q.copy_(qs[s]), kn.copy_(kns[s]), vn.copy_(vns[s])
        graph.replay()
        torch.cuda.synchronize()
        for b in range(batch):
            hold[b] = [np.concatenate([rows, _f64(x[s, b])[:, None]], 1) for rows, x in zip(hold[b], (kns, vns))]
            n = hold[b][0].shape[1]
            assert int(lens[b]) == n
            ref, ref_lse, mass, span = O.attend(_f64(q[b]), hold[b][0], hold[b][1], np.ones(n, bool), dh ** -0.5)
            d = 2.0 ** -23 * (dh + 4) * span
            assert (np.abs(_f64(o[b]) - ref) <= 2.0 ** -8 * np.abs(ref) + (2 * d + 2.0 ** -15 + 2.0 ** -22 * n)[:, None] * mass).all()
    assert int(status) == 0
    # a finished request gives its pages back; the table's other rows stay
    ends = _i32([int(lens[0]), -1, int(lens[2])])
    before = int(n_free)
    L.assign_pages(ends, table, free, n_free, page_size=page, held=lens, status=status, workspace=ws)
    assert lens.tolist()[1] == -1 and int(n_free) == before + -(-43 // page) and int(status) == 0
    plan.close()
