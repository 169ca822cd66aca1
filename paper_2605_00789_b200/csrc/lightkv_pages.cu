// Pages and rows of a serving cache: lightkv_assign_pages (block tables and slots from request lengths) and lightkv_append_kv
// (rows of new tokens to their slots).
//
// assign_pages.  With gone_b / grow_b the pages that request b gives back / asks for and G, T their exclusive prefix sums, the
// stack after the pushes holds at place i the free page i (i < n_free) or the released page i - n_free, and the k-th page asked
// for is the entry S - 1 - k of the S = n_free + sum(gone) there are.  So every page number that changes hands is found from
// its place alone: a moved page is read once where it stands now (a free entry, or the table row of a request that shrinks) and
// written once where it belongs (the stack above n_free, or the row of a request that grows).  Neither side touches what the
// other reads: entries above n_free are written only if no free page is taken.
// What is left is latency.  Few slots and up to kPageRows requests: a cluster whose CTAs all find the sums, so that none waits for
// another's, and share the moves; the first one writes the lengths, once all have read theirs (they may be the same array).
// Else one CTA finds the sums and a second kernel over the whole GPU moves pages and writes slots.
//   us a call on the device: 256 requests that grow by a token 4.5 -> 3.3, 64 that give back half of 65 pages on average 6.5 -> 3.4 (one
//   CTA of 1024 threads -> the cluster), 128 that are admitted with 438 000 slots 12.4 -> 8.6 (a slot a thread, rows searched in L2 ->
//   four, in shared memory).  Of 3.3 us, 1.4 are what any kernel takes in a row of dependent ones.
#include <limits.h>

#include "launch.h"
#include "tc_common.cuh"

namespace lkv {

namespace {

// Threads of a CTA; each looks at up to kPerThread requests (with a request a thread, 1024 threads, the shuffles of the sums alone
// took a microsecond of the SM).
constexpr int kPageThreads = 256, kPerThread = 4;
constexpr int kPageRows = kPageThreads * kPerThread;         // requests that are summed at once, and whose rows are kept on chip
constexpr int kPageCluster = 8;
constexpr int kPageSlots = 4096;       // most slots a cluster writes (569 slots 3.1 us against 4.1 with two kernels, 2084 4.2 : 4.3, 10084 4.6 : 4.4)

struct PageArgs {
  int batch, page_size, max_blocks, n_pages, add;
  unsigned page_mul; int page_shift;   // n / page_size = (umulhi(n, page_mul) + n) >> page_shift for n < 2^31
  const int* held; const int* seq_len;
  int* seq_len_out; int* block_table; int* free_pages;
  const int* n_free; int* n_free_out;
  long long* slot_map;
  int n_slots, slot_stride;
  int* slot_start;
  uint32_t* status;
  unsigned char* workspace;
};

__device__ __forceinline__ unsigned pages_of(const PageArgs& a, unsigned n) { return (__umulhi(n, a.page_mul) + n) >> a.page_shift; }   // whole ones

struct PageTotals { long long fresh; unsigned n_free, stacked, left, taken; };
// What is kept of the requests, in shared memory or in the workspace.  (The host has seen to it that all blocks of the table are
// counted in 32 bits.)
struct PageRows {
  long long* fresh_at;                 // exclusive sums of the new tokens asked for, and behind the last the whole
  unsigned *gone_at, *grow_at;         // exclusive sums of the pages given back and asked for
  int *held, *have, *need;             // tokens; pages held; pages afterwards (have and ~have where it was not served)
  __host__ __device__ static constexpr size_t bytes(int batch) { return (size_t(batch + 1) * 8 + size_t(batch) * 20 + 15) / 16 * 16; }
  __device__ __forceinline__ PageRows(unsigned char* p, int batch) {
    fresh_at = reinterpret_cast<long long*>(p);
    gone_at = reinterpret_cast<unsigned*>(fresh_at + batch + 1);
    grow_at = gone_at + batch;
    held = reinterpret_cast<int*>(grow_at + batch);
    have = held + batch;
    need = have + batch;
  }
};

struct Sums { long long fresh; unsigned gone, grow; };
__device__ __forceinline__ Sums add(const Sums& a, const Sums& b) { return {a.fresh + b.fresh, a.gone + b.gone, a.grow + b.grow}; }
__device__ __forceinline__ Sums scan(Sums a) {               // inclusive, over a warp
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums o = {__shfl_up_sync(0xffffffffu, a.fresh, d), __shfl_up_sync(0xffffffffu, a.gone, d), __shfl_up_sync(0xffffffffu, a.grow, d)};
    if (int(threadIdx.x & 31) >= d) a = add(a, o);
  }
  return a;
}

struct Request { int held, have, need, base; long long want; bool fits; };
__device__ __forceinline__ Sums page_request(const PageArgs& a, int b, Request& r, unsigned& status) {
  const int room = a.max_blocks * a.page_size;
  r.held = a.held ? max(a.held[b], 0) : 0;
  r.base = a.seq_len[b];
  r.want = r.base < 0 ? 0 : (long long)r.base + a.add;
  if (r.held > room) { r.held = room; status |= LIGHTKV_STATUS_COUNT; }
  r.have = r.held ? pages_of(a, r.held - 1) + 1 : 0;
  r.fits = r.want <= room;
  if (!r.fits) status |= LIGHTKV_STATUS_COUNT;
  r.need = r.fits ? (r.want ? pages_of(a, unsigned(r.want) - 1u) + 1 : 0) : r.have;
  return {max(r.want - r.held, 0ll), unsigned(max(r.have - r.need, 0)), unsigned(max(r.need - r.have, 0))};
}

// The sums over all requests, their rows, lengths and offsets, and the new height of the stack.  All threads of one CTA; `before`
// is called when everything has been read and before anything that a caller may have given as input is written, which
// `writes` CTAs do.
template <typename F>
__device__ void plan_pages(const PageArgs& a, const PageRows& rows, PageTotals& totals, bool writes, F before) {
  constexpr int WARPS = kPageThreads / 32;
  __shared__ Sums warp_sum[2][WARPS];
  __shared__ unsigned long long shared_max;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const bool chunks = a.batch > kPageRows;
  const int per = chunks ? kPerThread : (a.batch + kPageThreads - 1) / kPageThreads;         // consecutive requests of a thread
  unsigned status = 0;
  int n = *a.n_free;
  Request r[kPerThread];
  Sums own[kPerThread];
  auto read = [&](int b0) {
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      const int b = b0 + t * per + j;
      own[j] = {0, 0, 0};
      if (j < per && b < a.batch) own[j] = page_request(a, b, r[j], status);
    }
  };
  if (!chunks) {
    read(0);
    if (a.slot_map)                    // the pages of the next tokens, which slots may want
#pragma unroll
      for (int j = 0; j < kPerThread; ++j)
        if (j < per && t * per + j < a.batch && own[j].fresh > 0 && r[j].held < a.max_blocks * a.page_size)
          prefetch_l2(a.block_table + (size_t)(t * per + j) * a.max_blocks + pages_of(a, r[j].held));
  }
  if (n < 0 || n > a.n_pages) { n = n < 0 ? 0 : a.n_pages; status |= LIGHTKV_STATUS_COUNT; }
  const unsigned n_free = n;
  if (t < 32 && 32 * t < int(n_free)) prefetch_l2(a.free_pages + n_free - 1 - 32 * t);       // what is popped first
  unsigned stacked = 0;
  if (chunks) {                        // the height of the stack is needed before the first chunk
    unsigned gone = 0;
    for (int b = t; b < a.batch; b += kPageThreads) {
      unsigned ignore = 0;
      Request q;
      gone += page_request(a, b, q, ignore).gone;
    }
    gone = __reduce_add_sync(0xffffffffu, gone);
    if (t == 0) shared_max = 0;
    __syncthreads();
    if (lane == 0) atomicAdd(&shared_max, (unsigned long long)gone);
    __syncthreads();
    stacked = n_free + unsigned(shared_max);
    __syncthreads();
  }
  Sums carry = {0, 0, 0};
  unsigned taken = 0;
  int flip = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kPageRows, flip ^= 1) {
    if (chunks) read(b0);
    Sums mine = own[0];
#pragma unroll
    for (int j = 1; j < kPerThread; ++j) mine = add(mine, own[j]);
    const Sums sum = scan(mine);
    if (lane == 31) warp_sum[flip][warp] = sum;
    __syncthreads();
    Sums at = {carry.fresh + sum.fresh - mine.fresh, carry.gone + sum.gone - mine.gone, carry.grow + sum.grow - mine.grow}, chunk = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
      const Sums w = warp_sum[flip][i];
      if (i < warp) at = add(at, w);
      chunk = add(chunk, w);
    }
    if (!chunks) {
      stacked = n_free + chunk.gone;
      before();
    }
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      const int b = b0 + t * per + j;
      if (j >= per || b >= a.batch) break;
      const Sums next = add(at, own[j]);
      const bool served = r[j].fits && (own[j].grow == 0 || next.grow <= stacked);
      if (r[j].fits && !served) status |= LIGHTKV_STATUS_NO_PAGES;
      if (own[j].grow > 0 && served) taken = next.grow;      // the last one served has the largest
      rows.fresh_at[b] = at.fresh;
      rows.gone_at[b] = at.gone;
      rows.grow_at[b] = at.grow;
      rows.held[b] = r[j].held;
      rows.have[b] = r[j].have;
      rows.need[b] = served ? r[j].need : ~r[j].have;
      if (b == a.batch - 1) rows.fresh_at[a.batch] = next.fresh;
      if (writes) {
        a.seq_len_out[b] = r[j].base < 0 ? r[j].base : served ? (int)r[j].want : r[j].held;
        if (a.slot_start) {
          a.slot_start[b] = (int)min(at.fresh, (long long)INT_MAX);
          if (b == a.batch - 1) a.slot_start[a.batch] = (int)min(next.fresh, (long long)INT_MAX);
        }
        if (a.slot_map && own[j].fresh > 0) {
          const long long end = a.slot_stride ? (long long)b * a.slot_stride + min(own[j].fresh, (long long)a.slot_stride) : next.fresh;
          if (end > a.n_slots || (a.slot_stride && own[j].fresh > a.slot_stride)) status |= LIGHTKV_STATUS_COUNT;
        }
      }
      at = next;
    }
    carry = add(carry, chunk);
  }
  if (carry.grow <= stacked && !chunks) {
    taken = carry.grow;                // all were served (the others ask for nothing)
    __syncthreads();
  } else {
    taken = __reduce_max_sync(0xffffffffu, taken);
    if (t == 0) shared_max = 0;
    __syncthreads();
    if (lane == 0) atomicMax(&shared_max, (unsigned long long)taken);
    __syncthreads();
    taken = unsigned(shared_max);
  }
  unsigned left = stacked - taken;
  if (left > unsigned(a.n_pages)) { left = a.n_pages; status |= LIGHTKV_STATUS_COUNT; }      // page numbers held twice
  totals = {carry.fresh, n_free, stacked, left, taken};      // (in every thread)
  if (writes) {
    if (t == 0) *a.n_free_out = (int)left;
    if (a.status && status) atomicOr(a.status, status);
  }
}

// last row whose sum is at most `at`: the one that entry `at` belongs to
template <typename T>
__device__ __forceinline__ int find_row(const T* sums, int batch, T at) {
  int lo = 0, hi = batch;              // sums[lo] <= at < sums[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int released_page(const PageArgs& a, const PageRows& rows, unsigned i) {
  const int b = find_row(rows.gone_at, a.batch, i);
  const unsigned need = rows.need[b] < 0 ? ~rows.need[b] : rows.need[b], at = need + (i - rows.gone_at[b]);
  return at < unsigned(a.max_blocks) ? a.block_table[(size_t)b * a.max_blocks + at] : -1;
}
// the k-th page that is taken
__device__ __forceinline__ int taken_page(const PageArgs& a, const PageRows& rows, const PageTotals& s, unsigned k) {
  const unsigned i = s.stacked - 1 - k;
  return i < s.n_free ? a.free_pages[i] : released_page(a, rows, i - s.n_free);
}

// The moves and the slots, shared by `threads` threads of which this is number `id`.
__device__ void move_pages(const PageArgs& a, const PageRows& rows, const PageTotals& s, unsigned id, unsigned threads) {
  unsigned status = 0;
  if (a.slot_map) {
    // a thread writes `per` consecutive slots, which mostly lie in one page
    const int per = a.n_slots > int(threads) ? 4 : 1;
    const bool wide = per == 4 && (reinterpret_cast<uintptr_t>(a.slot_map) & 15) == 0;
    for (long long t0 = (long long)id * per; t0 < a.n_slots; t0 += (long long)threads * per) {
      long long slots[4];
      int b = -1, page = -1;
      unsigned at = 0xffffffffu;       // block of `page`
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long t = t0 + j;
        slots[j] = -1;
        if (j >= per) continue;
        long long i = 0;
        const int before = b;
        if (a.slot_stride) {
          b = int(unsigned(t) / unsigned(a.slot_stride));
          i = t - (long long)b * a.slot_stride;
        } else if (t < s.fresh) {
          if (b < 0) b = find_row(rows.fresh_at, a.batch, t);
          while (rows.fresh_at[b + 1] <= t) ++b;
          i = t - rows.fresh_at[b];
        } else {
          b = a.batch;
        }
        if (b >= a.batch || rows.need[b] < 0 || i >= rows.fresh_at[b + 1] - rows.fresh_at[b]) continue;
        const unsigned p = unsigned(rows.held[b]) + unsigned(i), block = pages_of(a, p);
        if (b != before || block != at)
          page = (int)block < rows.have[b] ? a.block_table[(size_t)b * a.max_blocks + block]
                                           : taken_page(a, rows, s, rows.grow_at[b] + (block - rows.have[b]));
        at = block;
        if (unsigned(page) < unsigned(a.n_pages)) slots[j] = (long long)page * a.page_size + (p - block * a.page_size);
        else status |= LIGHTKV_STATUS_PAGE;
      }
      if (wide && t0 + 4 <= a.n_slots) {
        reinterpret_cast<longlong2*>(a.slot_map + t0)[0] = make_longlong2(slots[0], slots[1]);
        reinterpret_cast<longlong2*>(a.slot_map + t0)[1] = make_longlong2(slots[2], slots[3]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < per && t0 + j < a.n_slots) a.slot_map[t0 + j] = slots[j];
      }
    }
  }
  id = threads - 1 - id;               // (pages move while others write slots)
  for (unsigned i = s.n_free + id; i < s.left; i += threads) a.free_pages[i] = released_page(a, rows, i - s.n_free);
  for (unsigned k = id; k < s.taken; k += threads) {
    const int b = find_row(rows.grow_at, a.batch, k);
    a.block_table[(size_t)b * a.max_blocks + rows.have[b] + (k - rows.grow_at[b])] = taken_page(a, rows, s, k);
  }
  if (status && a.status) atomicOr(a.status, status);
}

__global__ void __launch_bounds__(kPageThreads) pages_kernel(const __grid_constant__ PageArgs a) {
  __shared__ __align__(8) unsigned char on_chip[PageRows::bytes(kPageRows)];
  grid_dependency_sync();
  const PageRows rows(on_chip, a.batch);
  const unsigned rank = tc::cluster_ctarank();
  PageTotals totals;
  plan_pages(a, rows, totals, rank == 0, [&] {               // (what was read has arrived: nothing to release)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (rank == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  });
  move_pages(a, rows, totals, rank * kPageThreads + threadIdx.x, kPageCluster * kPageThreads);
  if (rank != 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(kPageThreads) pages_plan_kernel(const __grid_constant__ PageArgs a) {
  grid_dependency_sync();
  PageTotals totals;
  plan_pages(a, PageRows(a.workspace + 256, a.batch), totals, true, [] {});
  if (threadIdx.x == 0) *reinterpret_cast<PageTotals*>(a.workspace) = totals;
}

__global__ void __launch_bounds__(256) pages_move_kernel(const __grid_constant__ PageArgs a) {
  __shared__ __align__(16) unsigned char on_chip[PageRows::bytes(kPageRows)];
  grid_dependency_sync();
  unsigned char* from = a.workspace + 256;
  const PageTotals totals = *reinterpret_cast<const PageTotals*>(a.workspace);
  if (a.batch <= kPageRows) {
    const int pieces = int(PageRows::bytes(a.batch) / 16);   // (at most seven a thread, all asked for at once)
#pragma unroll
    for (int i = 0; i < int((PageRows::bytes(kPageRows) / 16 + 255) / 256); ++i)
      if (int(threadIdx.x) + i * 256 < pieces)
        tc::cp_async16(tc::smem_u32(on_chip) + (threadIdx.x + i * 256) * 16, from + (threadIdx.x + i * 256) * 16, 16);
    tc::cp_async_commit();
    tc::cp_async_wait<0>();
    __syncthreads();
    from = on_chip;
  }
  move_pages(a, PageRows(from, a.batch), totals, blockIdx.x * 256u + threadIdx.x, gridDim.x * 256u);
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

// A CTA copies `per_cta` tokens, all heads of K and V, four pieces in flight per thread.  Bound by HBM: 32768 rows of 8 heads x 128
// channels 45.0 us, 6.0 TB/s of reads and writes (the copy rate measured for the card is 6.56); 64 rows 1.4 us, a launch.
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

size_t lightkv_pages_workspace(int32_t batch) { return batch < 0 ? 0 : 256 + PageRows::bytes(batch); }

int lightkv_assign_pages(const lightkv_pages_args_t* a) {
  if (!a || a->struct_size != sizeof(lightkv_pages_args_t)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->batch <= 0 || a->page_size <= 0 || a->max_blocks <= 0 || a->n_pages <= 0 || a->add < 0 || a->n_slots < 0 || a->slot_stride < 0)
    return LIGHTKV_ERR_INVALID_ARG;
  if (!a->seq_len || !a->seq_len_out || !a->block_table || !a->free_pages || !a->n_free || !a->n_free_out || !a->workspace)
    return LIGHTKV_ERR_INVALID_ARG;
  if ((long long)a->max_blocks * a->page_size > INT_MAX) return LIGHTKV_ERR_INVALID_ARG;     // lengths are 32-bit
  if ((long long)a->max_blocks * a->batch + a->n_pages > INT_MAX) return LIGHTKV_ERR_UNSUPPORTED;            // pages are counted in 32 bits
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
  p.workspace = static_cast<unsigned char*>(a->workspace);
  page_divider((unsigned)a->page_size, &p.page_mul, &p.page_shift);
  cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  if (a->n_slots <= kPageSlots && a->batch <= kPageRows)
    return launch_kernel(pages_kernel, dim3(kPageCluster), dim3(kPageThreads), 0, stream, kPageCluster, p) == cudaSuccess ? LIGHTKV_OK : LIGHTKV_ERR_CUDA;
  if (launch_kernel(pages_plan_kernel, dim3(1), dim3(kPageThreads), 0, stream, 1, p) != cudaSuccess ||
      launch_kernel(pages_move_kernel, dim3(4u * sm_count()), dim3(256), 0, stream, 1, p) != cudaSuccess)
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
