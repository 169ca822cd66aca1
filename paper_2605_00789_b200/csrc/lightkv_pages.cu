// Pages and rows of a serving cache: lightkv_assign_pages (block tables and slots from request lengths) and lightkv_append_kv
// (rows of new tokens to their slots).
//
// assign_pages.  With gone_b / grow_b the pages that request b gives back / asks for and G, T their exclusive prefix sums, the
// stack after the pushes holds at place i the free page i (i < n_free) or the released page i - n_free, and the k-th page asked
// for is the entry S - 1 - k of the S = n_free + sum(gone) there are.  So every page number that changes hands is found from
// its place alone: a moved page is read once where it stands now (a free entry, or the table row of a request that shrinks) and
// written once where it belongs (the stack above n_free, or the row of a request that grows).  Neither side touches what the
// other reads: entries above n_free are written only if no free page is taken.
// One CTA finds the sums (a few microseconds of latency); with few slots it also moves the pages and writes the slots, else a
// second kernel over the whole GPU does.
#include <limits.h>

#include "launch.h"

namespace lkv {

namespace {

struct PageRow {                       // one request
  int held, have, need;                // tokens; pages held, pages afterwards (have where it was not served)
  int served;
  long long gone_at, grow_at, fresh_at;          // exclusive prefix sums over the requests in front
  long long fresh;                     // new tokens asked for
};
struct PageTotals { long long n_free, stacked, left, taken, fresh; };

constexpr int kPageThreads = 1024;
constexpr int kPageRowsOnChip = 768;   // requests whose rows fit the shared memory a CTA has without asking
constexpr size_t kTotalsBytes = 256;

struct PageArgs {
  int batch, page_size, max_blocks, n_pages, add;
  const int* held; const int* seq_len;
  int* seq_len_out; int* block_table; int* free_pages;
  const int* n_free; int* n_free_out;
  long long* slot_map;
  int n_slots, slot_stride;
  int* slot_start;
  uint32_t* status;
  PageRow* rows;                       // workspace
  PageTotals* totals;
};

struct Sums { long long gone, grow, fresh; };
__device__ __forceinline__ Sums add(const Sums& a, const Sums& b) { return {a.gone + b.gone, a.grow + b.grow, a.fresh + b.fresh}; }
__device__ __forceinline__ Sums shfl_up(const Sums& a, int d) {
  return {__shfl_up_sync(0xffffffffu, a.gone, d), __shfl_up_sync(0xffffffffu, a.grow, d), __shfl_up_sync(0xffffffffu, a.fresh, d)};
}

// What request b asks for; `status` collects its complaints.
__device__ __forceinline__ Sums page_request(const PageArgs& a, int b, PageRow& r, long long& want, int& base, unsigned& status) {
  const long long room = (long long)a.max_blocks * a.page_size;
  long long held = a.held ? max(a.held[b], 0) : 0;
  base = a.seq_len[b];
  want = base < 0 ? 0 : (long long)base + a.add;
  if (held > room) { held = room; status |= LIGHTKV_STATUS_COUNT; }
  r.held = (int)held;
  r.have = (int)((held + a.page_size - 1) / a.page_size);
  r.fresh = max(want - held, 0ll);
  r.served = want <= room;
  if (!r.served) status |= LIGHTKV_STATUS_COUNT;
  r.need = r.served ? (int)((want + a.page_size - 1) / a.page_size) : r.have;
  return {max(r.have - r.need, 0), max(r.need - r.have, 0), r.fresh};
}

// The sums over all requests, their rows, lengths and offsets, and the new height of the stack.  All threads of one CTA.
__device__ void plan_pages(const PageArgs& a, PageRow* rows, PageTotals* totals) {
  __shared__ Sums warp_sum[32];
  __shared__ long long all_gone;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  unsigned status = 0;
  long long n_free = *a.n_free;
  if (n_free < 0 || n_free > a.n_pages) { n_free = n_free < 0 ? 0 : a.n_pages; status |= LIGHTKV_STATUS_COUNT; }
  Sums carry = {0, 0, 0};
  long long stacked = 0, taken = 0;
  if (a.batch > kPageThreads) {        // the height of the stack is needed before the first chunk
    long long gone = 0;
    for (int b = t; b < a.batch; b += kPageThreads) {
      PageRow r; long long want; int base; unsigned ignore = 0;
      gone += page_request(a, b, r, want, base, ignore).gone;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) gone += __shfl_xor_sync(0xffffffffu, gone, d);
    if (t == 0) all_gone = 0;
    __syncthreads();
    if (lane == 0) atomicAdd(reinterpret_cast<unsigned long long*>(&all_gone), (unsigned long long)gone);
    __syncthreads();
    stacked = n_free + all_gone;
  }
  for (int b0 = 0; b0 < a.batch; b0 += kPageThreads) {
    const int b = b0 + t;
    PageRow r = {};
    long long want = 0;
    int base = 0;
    Sums own = {0, 0, 0};
    if (b < a.batch) own = page_request(a, b, r, want, base, status);
    Sums sum = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const Sums o = shfl_up(sum, d);
      if (lane >= d) sum = add(sum, o);
    }
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      Sums v = warp_sum[lane];
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const Sums o = shfl_up(v, d);
        if (lane >= d) v = add(v, o);
      }
      warp_sum[lane] = v;
    }
    __syncthreads();
    const Sums chunk = warp_sum[31];
    sum = add(sum, carry);
    if (warp > 0) sum = add(sum, warp_sum[warp - 1]);        // inclusive, over all requests
    if (a.batch <= kPageThreads) stacked = n_free + chunk.gone;
    if (b < a.batch) {
      const bool short_of = own.grow > 0 && sum.grow > stacked;
      if (short_of) { status |= LIGHTKV_STATUS_NO_PAGES; r.served = 0; r.need = r.have; }
      r.gone_at = sum.gone - own.gone;
      r.grow_at = sum.grow - own.grow;
      r.fresh_at = sum.fresh - own.fresh;
      if (own.grow > 0 && !short_of) taken = sum.grow;       // the last one served has the largest
      rows[b] = r;
      a.seq_len_out[b] = base < 0 ? base : r.served ? (int)want : r.held;
      if (a.slot_start) {
        a.slot_start[b] = (int)min(r.fresh_at, (long long)INT_MAX);
        if (b == a.batch - 1) a.slot_start[a.batch] = (int)min(sum.fresh, (long long)INT_MAX);
      }
      if (a.slot_map) {
        const long long end = a.slot_stride ? (long long)b * a.slot_stride + min(r.fresh, (long long)a.slot_stride) : sum.fresh;
        if (r.fresh > 0 && (end > a.n_slots || (a.slot_stride && r.fresh > a.slot_stride))) status |= LIGHTKV_STATUS_COUNT;
      }
    }
    carry = add(carry, chunk);
    __syncthreads();
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) taken = max(taken, __shfl_xor_sync(0xffffffffu, taken, d));
  if (t == 0) all_gone = 0;
  __syncthreads();
  if (lane == 0) atomicMax(reinterpret_cast<unsigned long long*>(&all_gone), (unsigned long long)taken);
  __syncthreads();
  taken = all_gone;
  if (t == 0) {
    long long left = stacked - taken;
    if (left > a.n_pages) { left = a.n_pages; status |= LIGHTKV_STATUS_COUNT; }      // page numbers held twice
    *totals = {n_free, stacked, left, taken, carry.fresh};
    *a.n_free_out = (int)left;
  }
  if (a.status && status) atomicOr(a.status, status);
  __syncthreads();
}

// last request whose prefix sum is at most `at` among those with the sum non-decreasing: the one that entry `at` belongs to
template <typename Get>
__device__ __forceinline__ int find_row(int batch, long long at, Get get) {
  int lo = 0, hi = batch;              // get(lo) <= at < get(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (get(mid) <= at) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int released_page(const PageArgs& a, const PageRow* rows, long long i) {
  const int b = find_row(a.batch, i, [&](int m) { return rows[m].gone_at; });
  const long long at = rows[b].need + (i - rows[b].gone_at);
  return at < a.max_blocks ? a.block_table[(size_t)b * a.max_blocks + at] : -1;
}
// the k-th page that is taken
__device__ __forceinline__ int taken_page(const PageArgs& a, const PageRow* rows, const PageTotals& s, long long k) {
  const long long i = s.stacked - 1 - k;
  return i < s.n_free ? a.free_pages[i] : released_page(a, rows, i - s.n_free);
}

// The moves and the slots, shared by `threads` threads of which this is number `id`.
__device__ void move_pages(const PageArgs& a, const PageRow* rows, const PageTotals& s, long long id, long long threads) {
  for (long long i = s.n_free + id; i < s.left; i += threads) a.free_pages[i] = released_page(a, rows, i - s.n_free);
  for (long long k = id; k < s.taken; k += threads) {
    const int b = find_row(a.batch, k, [&](int m) { return rows[m].grow_at; });
    a.block_table[(size_t)b * a.max_blocks + rows[b].have + (k - rows[b].grow_at)] = taken_page(a, rows, s, k);
  }
  if (!a.slot_map) return;
  unsigned status = 0;
  for (long long t = id; t < a.n_slots; t += threads) {
    long long slot = -1, i = 0;
    int b = a.batch;
    if (a.slot_stride) {
      b = (int)(t / a.slot_stride);
      i = t - (long long)b * a.slot_stride;
    } else if (t < s.fresh) {
      b = find_row(a.batch, t, [&](int m) { return rows[m].fresh_at; });
      i = t - rows[b].fresh_at;
    }
    if (b < a.batch) {
      const PageRow& r = rows[b];
      if (r.served && i < r.fresh) {
        const unsigned p = unsigned(r.held) + unsigned(i), block = p / unsigned(a.page_size);
        const int page = (int)block < r.have ? a.block_table[(size_t)b * a.max_blocks + block]
                                             : taken_page(a, rows, s, r.grow_at + ((int)block - r.have));
        if (unsigned(page) < unsigned(a.n_pages)) slot = (long long)page * a.page_size + (p - block * a.page_size);
        else status |= LIGHTKV_STATUS_PAGE;
      }
    }
    a.slot_map[t] = slot;
  }
  if (status && a.status) atomicOr(a.status, status);
}

__global__ void __launch_bounds__(kPageThreads) pages_kernel(const __grid_constant__ PageArgs a) {
  __shared__ PageRow on_chip[kPageRowsOnChip];
  __shared__ PageTotals totals;
  grid_dependency_sync();
  PageRow* rows = a.batch <= kPageRowsOnChip ? on_chip : a.rows;
  plan_pages(a, rows, &totals);
  move_pages(a, rows, totals, threadIdx.x, kPageThreads);
}

__global__ void __launch_bounds__(kPageThreads) pages_plan_kernel(const __grid_constant__ PageArgs a) {
  grid_dependency_sync();
  plan_pages(a, a.rows, a.totals);
}

__global__ void __launch_bounds__(256) pages_move_kernel(const __grid_constant__ PageArgs a) {
  grid_dependency_sync();
  move_pages(a, a.rows, *a.totals, blockIdx.x * 256ll + threadIdx.x, gridDim.x * 256ll);
}

// ---- rows of new tokens ---------------------------------------------------------------------------------------------------
struct AppendArgs {
  const char* k_new; const char* v_new;
  char* k_cache; char* v_cache;
  int64_t new_token, new_head, page, head, row;    // bytes
  const long long* slot_map;
  uint32_t* status;
  long long n_slots;                   // of the pool
  int n_tokens, n_kv_heads, pieces;    // 16-byte pieces of a row
  int page_size;
  int per_cta;                         // tokens
  unsigned magic_token, magic_pieces;  // divisors: pieces of a token's K and V, pieces of a row (0: one piece)
};

// A CTA copies `per_cta` tokens, all heads of K and V, four pieces in flight per thread.
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendArgs a) {
  grid_dependency_sync();
  const int first = blockIdx.x * a.per_cta, n = min(a.per_cta, a.n_tokens - first);
  const int per_kv = a.n_kv_heads * a.pieces, per_token = 2 * per_kv, units = n * per_token;
  for (int u0 = threadIdx.x; u0 < units; u0 += 4 * 256) {
    uint4 v[4];
    char* to[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int u = u0 + q * 256;
      to[q] = nullptr;
      if (u < units) {
        const int t = div_magic(u, a.magic_token), rem = u - t * per_token, kv = rem >= per_kv ? 1 : 0, piece = rem - kv * per_kv;
        const int h = a.magic_pieces ? div_magic(piece, a.magic_pieces) : piece, c = piece - h * a.pieces;
        const long long slot = a.slot_map[first + t];
        if (slot >= 0 && slot < a.n_slots) {
          const long long page = slot / a.page_size;
          to[q] = (kv ? a.v_cache : a.k_cache) + page * a.page + (slot - page * a.page_size) * a.row + h * a.head + c * 16;
          v[q] = ld_stream16((kv ? a.v_new : a.k_new) + (first + t) * a.new_token + h * a.new_head + c * 16);
        } else if (slot >= 0 && rem == 0 && a.status) {
          atomicOr(a.status, LIGHTKV_STATUS_PAGE);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (to[q]) st_stream16(to[q], v[q]);
  }
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

}  // namespace lkv

using namespace lkv;

extern "C" {

size_t lightkv_pages_workspace(int32_t batch) { return batch < 0 ? 0 : kTotalsBytes + size_t(batch) * sizeof(PageRow); }

int lightkv_assign_pages(const lightkv_pages_args_t* a) {
  if (!a || a->struct_size != sizeof(lightkv_pages_args_t)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->batch <= 0 || a->page_size <= 0 || a->max_blocks <= 0 || a->n_pages <= 0 || a->add < 0 || a->n_slots < 0 || a->slot_stride < 0)
    return LIGHTKV_ERR_INVALID_ARG;
  if (!a->seq_len || !a->seq_len_out || !a->block_table || !a->free_pages || !a->n_free || !a->n_free_out || !a->workspace)
    return LIGHTKV_ERR_INVALID_ARG;
  if ((long long)a->max_blocks * a->page_size > INT_MAX) return LIGHTKV_ERR_INVALID_ARG;     // lengths are 32-bit
  if (!a->slot_map != !a->n_slots || (a->slot_stride && !a->slot_map)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->slot_map && !aligned(a->slot_map, 8)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->block_table == a->free_pages || a->seq_len_out == a->n_free_out || a->seq_len_out == a->slot_start) return LIGHTKV_ERR_INVALID_ARG;
  if (!aligned(a->workspace, 256) || a->workspace_bytes < lightkv_pages_workspace(a->batch)) return LIGHTKV_ERR_WORKSPACE;
  PageArgs p = {};
  p.batch = a->batch; p.page_size = a->page_size; p.max_blocks = a->max_blocks; p.n_pages = a->n_pages; p.add = a->add;
  p.held = a->held; p.seq_len = a->seq_len; p.seq_len_out = a->seq_len_out; p.block_table = a->block_table;
  p.free_pages = a->free_pages; p.n_free = a->n_free; p.n_free_out = a->n_free_out;
  p.slot_map = reinterpret_cast<long long*>(a->slot_map); p.n_slots = a->n_slots; p.slot_stride = a->slot_stride;
  p.slot_start = a->slot_start; p.status = a->status;
  p.totals = static_cast<PageTotals*>(a->workspace);
  p.rows = reinterpret_cast<PageRow*>(static_cast<char*>(a->workspace) + kTotalsBytes);
  cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  if (a->n_slots <= 4 * kPageThreads && a->batch <= kPageRowsOnChip)
    return launch_kernel(pages_kernel, dim3(1), dim3(kPageThreads), 0, stream, 1, p) == cudaSuccess ? LIGHTKV_OK : LIGHTKV_ERR_CUDA;
  const unsigned grid = 4u * sm_count();
  if (launch_kernel(pages_plan_kernel, dim3(1), dim3(kPageThreads), 0, stream, 1, p) != cudaSuccess ||
      launch_kernel(pages_move_kernel, dim3(grid), dim3(256), 0, stream, 1, p) != cudaSuccess)
    return LIGHTKV_ERR_CUDA;
  return LIGHTKV_OK;
}

int lightkv_append_kv(const lightkv_append_args_t* a) {
  if (!a || a->struct_size != sizeof(lightkv_append_args_t)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->n_tokens < 0 || a->n_kv_heads <= 0 || a->head_dim <= 0 || a->head_dim % 8 || a->page_size <= 0 || a->n_pages <= 0 ||
      (a->dtype != LIGHTKV_BF16 && a->dtype != LIGHTKV_FP32))
    return LIGHTKV_ERR_INVALID_ARG;
  if (a->head_dim > 256) return LIGHTKV_ERR_UNSUPPORTED;
  const int el = a->dtype == LIGHTKV_BF16 ? 2 : 4, pieces = a->head_dim * el / 16;
  if ((long long)a->n_kv_heads * pieces * 2 > 32767) return LIGHTKV_ERR_UNSUPPORTED;         // 16-bit piece numbers
  if (!a->k_cache || !a->v_cache || (a->n_tokens > 0 && (!a->k_new || !a->v_new || !a->slot_map))) return LIGHTKV_ERR_INVALID_ARG;
  const void* ptrs[4] = {a->k_new, a->v_new, a->k_cache, a->v_cache};
  for (const void* p : ptrs) if (!aligned(p, 16)) return LIGHTKV_ERR_INVALID_ARG;
  const int64_t strides[5] = {a->new_token_stride, a->new_head_stride, a->page_stride, a->head_stride, a->row_stride};
  for (int64_t s : strides) if (s * el % 16) return LIGHTKV_ERR_INVALID_ARG;
  if (a->row_stride < a->head_dim || a->k_cache == a->v_cache || a->k_new == a->k_cache || a->v_new == a->v_cache) return LIGHTKV_ERR_INVALID_ARG;
  if (a->n_tokens == 0) return LIGHTKV_OK;
  AppendArgs p = {};
  p.k_new = static_cast<const char*>(a->k_new); p.v_new = static_cast<const char*>(a->v_new);
  p.k_cache = static_cast<char*>(a->k_cache); p.v_cache = static_cast<char*>(a->v_cache);
  p.new_token = a->new_token_stride * el; p.new_head = a->new_head_stride * el;
  p.page = a->page_stride * el; p.head = a->head_stride * el; p.row = a->row_stride * el;
  p.slot_map = reinterpret_cast<const long long*>(a->slot_map); p.status = a->status;
  p.n_slots = (long long)a->n_pages * a->page_size;
  p.n_tokens = a->n_tokens; p.n_kv_heads = a->n_kv_heads; p.pieces = pieces; p.page_size = a->page_size;
  const int per_token = 2 * a->n_kv_heads * pieces;
  // a token per CTA while the SMs are not full, else 2048 pieces
  p.per_cta = a->n_tokens <= 4 * sm_count() || per_token >= 2048 ? 1 : 2048 / per_token;
  p.magic_token = div_multiplier(per_token);
  p.magic_pieces = pieces > 1 ? div_multiplier(pieces) : 0;
  const unsigned grid = (unsigned)((a->n_tokens + p.per_cta - 1) / p.per_cta);
  if (launch_kernel(append_kernel, dim3(grid), dim3(256), 0, static_cast<cudaStream_t>(a->stream), 1, p) != cudaSuccess)
    return LIGHTKV_ERR_CUDA;
  return LIGHTKV_OK;
}

}  // extern "C"
