// Attention of one new token per request over a paged (or contiguous) cache: lightkv_decode_attention.
//
//   out = softmax(scale q K^T) V  per (request, query head),  lse = log sum exp(scale q K^T)
//
// Every key and value is read once and used for two dot products per query head, so the pass is bound by HBM wherever the
// query heads of a key head share the read.  A warp walks its own pieces of 16 keys through its own ring of cp.async stages and
// keeps the running maximum and sum of the softmax; no barrier stands between warps before the end.  What has to be kept
// low is the latency of a piece's arithmetic: a warp that computes longer than its ring's copies take leaves HBM idle.
//
// bf16: keys are the rows of the first product (S^T = K Q^T, mma.sync m16n8k16: 16 keys x 8 query heads), channels the rows of
// the second (O^T = V^T P^T), so that eight query heads fill the narrow side of an MMA.  Rows lie in shared memory as they
// come, 16-byte units permuted by the row's last three bits; ldmatrix reads K as it is and V transposed.  P is rounded to two
// bf16 summands (hi + lo, 16 bits of mantissa): with one the rounding of P would be as large as the rounding of the output row.
// tcgen05 would need 64 rows of query heads to save arithmetic that HBM hides.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "decode_join.cuh"
#include "launch.h"
#include "tc_common.cuh"

namespace lkv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSms = 148;              // the workspace is sized for them
constexpr int kMaxCluster = 8;
constexpr int kPiece = 16;             // keys of a ring stage; a warp looks up the rows of two pieces at once, one per lane

struct DecodeArgs {
  const char* q; const char* k; const char* v; const char* k_new; const char* v_new;
  char* out;
  float* lse;
  const int* table;                    // nullptr: contiguous
  const int* n_keys;
  const long long* slot_map;           // nullptr: every request has a new row where k_new is given
  uint32_t* status;
  int64_t lse_batch, lse_head;         // elements
  // strides in units of 16 bytes
  uint32_t q_batch, q_head, page, head, row, new_batch, new_head, out_batch, out_head;
  int n_kv_heads, group, row_blocks, dh, page_size, max_blocks, n_pages;
  int cap;                             // rows a request has room for
  float scale_log2;
  unsigned page_mul; int page_shift;   // key / page_size = (umulhi(key, page_mul) + key) >> page_shift for key < 2^31
  int aligned;                         // pieces do not straddle pages
  int near_rows;                       // units of 16 bytes to any row fit 32 bits
};

using tc::cluster_sync;
using tc::smem_u32;

// i strides of 16-byte units, in bytes
__device__ __forceinline__ int64_t bytes_of(uint32_t i, uint32_t stride) { return int64_t((uint64_t(i) * stride) << 4); }
// 16 bytes, the first `bytes` of them from global memory, the rest zero; TO, FROM: constant offsets
template <int TO, int FROM>
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0+%3], [%1+%4], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(TO), "n"(FROM) : "memory");
}
// f(Const<0>) ... f(Const<N - 1>)
template <int I> struct Const { static constexpr int value = I; };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F f) {
  if constexpr (I < N) {
    f(Const<I>());
    unrolled<N, I + 1>(f);
  }
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// What a warp knows of one request and key head, and of the piece whose rows are looked up.
struct Walk {
  const char *k, *v;                   // the head's row 0 of page 0
  const char *k_new, *v_new;           // rows that stand for key n - 1, or nullptr
  const int* table;
  int n;                               // keys
  int first, step;                     // pieces first, first + step, ...
  // Page numbers are asked for long before they are needed.  Aligned: lane i holds that of the (32 j + i)-th piece, `ahead` those of
  // the next 32.  Else lanes 0 .. 15 hold those of the keys of an even piece, 16 .. 31 of the one behind it, `ahead` of the next two.
  int pages, ahead;
  int64_t off;                         // bytes to the row of key lane % 16 (aligned: of key 0) of the piece in hand
  unsigned mask;                       // bit i: key i of the piece in hand is there
  int own;                             // which of them the token's own row stands for, or -1
  bool bad;                            // a page number outside the pool was met

  __device__ __forceinline__ void start(const DecodeArgs& a, int b, int hk, int first_piece, int by) {
    table = a.table ? a.table + size_t(b) * a.max_blocks : nullptr;
    const int64_t at = bytes_of(hk, a.head) + (a.table ? 0 : bytes_of(b, a.page));
    k = a.k + at;
    v = a.v + at;
    k_new = v_new = nullptr;
    if (a.k_new) {
      const int64_t own_at = bytes_of(b, a.new_batch) + bytes_of(hk, a.new_head);
      k_new = a.k_new + own_at;
      v_new = a.v_new + own_at;
    }
    first = first_piece; step = by;
    bad = false;
  }
  // A request without a slot has no new row.  (Asked for behind the page numbers, which are needed first: with a slot map 1 x 404 keys
  // take 6.63 us and 24 x 90 .. 2000 of 64 channels 14.45, against 6.61 and 14.19 without; asked for in start() 7.0 and 14.8.)
  __device__ __forceinline__ void look_slot(const DecodeArgs& a, int b) {
    if (a.slot_map && a.slot_map[b] < 0) k_new = nullptr;
  }
  static __device__ __forceinline__ unsigned block_of(const DecodeArgs& a, unsigned key) { return (__umulhi(key, a.page_mul) + key) >> a.page_shift; }
  // this lane's page number among those looked up from the i-th piece on; -1 behind `limit` keys
  __device__ __forceinline__ int look_up(const DecodeArgs& a, int i, int limit) const {
    const unsigned lane = threadIdx.x & 31;
    const long long piece = first + (long long)(i + int(a.aligned ? lane : lane >> 4)) * step;
    const long long key = piece * kPiece + (a.aligned ? 0 : lane & 15);
    return key < limit ? table[block_of(a, unsigned(key))] : -1;
  }
  __device__ __forceinline__ void look(const DecodeArgs& a, int limit) {
    if (!table) return;
    pages = look_up(a, 0, limit);
    ahead = look_up(a, a.aligned ? 32 : 2, limit);
  }
  // rows of the i-th piece; called for i = 0, 1, 2, ...
  __device__ __forceinline__ void locate(const DecodeArgs& a, int i) {
    const unsigned lane = threadIdx.x & 31, key0 = unsigned(first + i * step) * kPiece, there = unsigned(n) - key0;
    mask = there >= kPiece ? 0xffffu : (1u << there) - 1u;
    own = k_new && there <= unsigned(kPiece) ? int(there) - 1 : -1;
    if (!table) {
      off = bytes_of(key0, a.row);
    } else if (a.aligned) {
      const int page = __shfl_sync(0xffffffffu, pages, i & 31);
      const bool in_pool = unsigned(page) < unsigned(a.n_pages);
      if (!in_pool) { mask = 0; bad = true; }
      off = in_pool ? bytes_of(page, a.page) + bytes_of(key0 - block_of(a, key0) * unsigned(a.page_size), a.row) : 0;
      if ((i & 31) == 31) {
        pages = ahead;
        ahead = look_up(a, i + 33, n);
      }
    } else {
      const int page = __shfl_sync(0xffffffffu, pages, (i & 1) * 16 + (lane & 15));
      const unsigned key = key0 + (lane & 15);
      const bool in_pool = unsigned(page) < unsigned(a.n_pages), ok = key < unsigned(n);
      bad |= ok && !in_pool;
      mask &= __ballot_sync(0xffffffffu, in_pool);
      off = ok && in_pool ? bytes_of(page, a.page) + bytes_of(key - block_of(a, key) * unsigned(a.page_size), a.row) : 0;
      if (i & 1) {
        pages = ahead;
        ahead = look_up(a, i + 3, n);
      }
    }
  }
};

// fp32, K: rows are copied in whole lines, 32 consecutive 16-byte units per instruction, and land where the lane that needs them
// reads them: unit x of row r belongs to lane 4 (r % 8) + x % 4 as its unit (r / 8) U / 4 + x / 4 of U.
// This lane's unit of row `odd` (0 or 1) of K lands there; 64 bytes further for every row further, 512 U / 4 behind eight.
__device__ __forceinline__ uint32_t k_lane(int odd) {
  const int lane = threadIdx.x & 31;
  return (lane / 4) * 512 + (((odd * 4 + lane % 4) ^ ((lane / 4 & 1) << 2)) * 16);
}
// the slot that a lane reads its K piece kc from
__device__ __forceinline__ int k_slot(int kc) { return (threadIdx.x & 31) ^ ((kc & 1) << 2); }

// Partial rows in shared memory, kRows x kWidth floats, each pair of rows turned by eight channels against the one before (so that
// the rows of a lane quad fall into different banks).
template <typename W>
struct Partial {
  static constexpr int kBytes = W::kRows * W::kWidth * 4;
  static __device__ __forceinline__ int at(int r, int d) { return r * W::kWidth + ((d + (r >> 1 & 3) * 8) & (W::kWidth - 1)); }
};

// ---- bf16 ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}

// DC: channels in units of 64 (0: 32 channels); NH: query heads in units of 8
template <int DC, int NH>
struct WarpBf16 {
  static constexpr int kRows = 8 * NH, kWidth = DC ? 64 * DC : 32, KC = kWidth / 16;       // KC: steps of 16 channels
  static constexpr int kRowBytes = kWidth * 2, kHalf = kPiece * kRowBytes;
  static constexpr int kStage = 2 * kHalf;                   // bytes: K, then V
  uint32_t q[NH][KC][2];
  float o[NH][KC][4];                  // channels 16 t + g (and + 8), heads 2c, 2c + 1 of lane 4 g + c
  float m[NH][2], l[NH][2];            // heads 2c and 2c + 1: reference exponent; this lane's part of the sum

  // unit x of row r lies at unit x ^ turn(r) of the row, so that a unit of eight rows in a row falls into all banks
  static __device__ __forceinline__ int turn(int r) { return kWidth >= 64 ? r & 7 : r >> 1 & 3; }
  // the query rows as 16-byte units, permuted as the stages' are
  static __device__ __forceinline__ uint32_t q_unit(int r, int x) { return r * kRowBytes + ((x ^ turn(r)) << 4); }
  __device__ __forceinline__ void load_q(const unsigned char* rows) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      // matrices of 8 heads x 8 channels: channels 0, 8, 16, 24 of two steps
      const uint32_t at = smem_u32(rows) + (h * 8 + (lane & 7)) * kRowBytes + (((lane >> 3) ^ turn(lane & 7)) << 4);
#pragma unroll
      for (int kc = 0; kc < KC; kc += 2) {
        uint32_t f[4];
        ldmatrix4(f, (at ^ (kc % 4 << 5)) + kc / 4 * 128);
        q[h][kc][0] = f[0]; q[h][kc][1] = f[1]; q[h][kc + 1][0] = f[2]; q[h][kc + 1][1] = f[3];
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int t = 0; t < KC; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[h][t][i] = 0.f;
      m[h][0] = m[h][1] = -INFINITY;
      l[h][0] = l[h][1] = 0.f;
    }
  }
  // Copy the piece in hand into the stage at `stage`.
  __device__ __forceinline__ void fetch(const DecodeArgs& a, const Walk& w, uint32_t stage) {
    constexpr int CH = kWidth / 8, R = 32 / CH, N = kPiece / R;              // units of a row; rows an instruction, instructions
    const int lane = threadIdx.x & 31, x = lane % CH, lr = lane / CH;
    const uint32_t dst = stage + lr * kRowBytes + ((x ^ turn(lr)) << 4);     // ^ ((n R) % 8 << 4), + n R kRowBytes
    const bool there = x * 8 < a.dh;
    if (a.aligned && w.mask == 0xffffu && w.own < 0) {
      const int64_t off = w.off + x * 16 + bytes_of(lr, a.row);
      const char *k = w.k + off, *v = w.v + off;
      if (a.dh == kWidth && a.row == kRowBytes / 16) {
        unrolled<N>([&](auto cn) {
          constexpr int r0 = decltype(cn)::value * R;
          copy16<r0 * kRowBytes, r0 * kRowBytes>(dst ^ (r0 % 8 << 4), k, 16);
          copy16<r0 * kRowBytes + kHalf, r0 * kRowBytes>(dst ^ (r0 % 8 << 4), v, 16);
        });
      } else {
        unrolled<N>([&](auto cn) {
          constexpr int r0 = decltype(cn)::value * R;
          copy16<r0 * kRowBytes, 0>(dst ^ (r0 % 8 << 4), k, there ? 16 : 0);
          copy16<r0 * kRowBytes + kHalf, 0>(dst ^ (r0 % 8 << 4), v, there ? 16 : 0);
          k += bytes_of(R, a.row);
          v += bytes_of(R, a.row);
        });
      }
      return;
    }
    if (a.near_rows && w.mask == 0xffffu && w.own < 0) {     // (unaligned: a row's units by one shuffle)
      const char *k = w.k + x * 16, *v = w.v + x * 16;
      const uint32_t units = uint32_t(w.off >> 4);
      unrolled<N>([&](auto cn) {
        constexpr int r0 = decltype(cn)::value * R;
        const uint64_t off = uint64_t(__shfl_sync(0xffffffffu, units, r0 + lr)) * 16;
        copy16<r0 * kRowBytes, 0>(dst ^ (r0 % 8 << 4), k + off, there ? 16 : 0);
        copy16<r0 * kRowBytes + kHalf, 0>(dst ^ (r0 % 8 << 4), v + off, there ? 16 : 0);
      });
      return;
    }
    unrolled<N>([&](auto cn) {
      constexpr int r0 = decltype(cn)::value * R;
      const int j = r0 + lr;
      const int64_t off = a.aligned ? w.off + bytes_of(j, a.row) : __shfl_sync(0xffffffffu, w.off, j);
      const int bytes = there && ((w.mask >> j) & 1) ? 16 : 0;
      copy16<r0 * kRowBytes, 0>(dst ^ (r0 % 8 << 4), (j == w.own ? w.k_new : w.k + off) + x * 16, bytes);
      copy16<r0 * kRowBytes + kHalf, 0>(dst ^ (r0 % 8 << 4), (j == w.own ? w.v_new : w.v + off) + x * 16, bytes);
    });
  }
  // 16 keys; bit i of `mask`: key i counts
  __device__ __forceinline__ void use(const DecodeArgs& a, const unsigned char* stage, unsigned mask) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const uint32_t at = smem_u32(stage);
    // K: matrices of 8 keys x 8 channels in the order (keys, channels) (0, 0), (8, 0), (0, 8), (8, 8)
    const uint32_t ka = at + (lane & 15) * kRowBytes + (((lane >> 4) ^ turn(lane & 7)) << 4);
    float s[NH][4], s2[NH][4];         // two chains of products
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[h][i] = s2[h][i] = 0.f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      uint32_t f[4];
      ldmatrix4(f, (ka ^ (kc % 4 << 5)) + kc / 4 * 128);
#pragma unroll
      for (int h = 0; h < NH; ++h) mma16816(kc & 1 ? s2[h] : s[h], f[0], f[1], f[2], f[3], q[h][kc][0], q[h][kc][1]);
    }
    // s[h][0], s[h][1]: key g, heads 2c and 2c + 1; s[h][2], s[h][3]: key g + 8
    bool grows = false;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[h][i] = (s[h][i] + s2[h][i]) * a.scale_log2;
        if (mask != 0xffffu && !((mask >> (g + (i >> 1) * 8)) & 1)) s[h][i] = -INFINITY;
        grows |= s[h][i] > m[h][i & 1] + 8.f;
      }
    // The reference of a row is raised only where a logit exceeds it by 2^8: weights stay below 256, sums in range.  It stays finite:
    // a logit of +inf has an infinite weight and sum (inf - inf would leave no number for lse).
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(s[h][e], s[h][2 + e]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          top = fminf(fmaxf(top, m[h][e]), FLT_MAX);
          const float f = top == -INFINITY ? 1.f : exp2_approx(m[h][e] - top);
          m[h][e] = top;
          l[h][e] *= f;
#pragma unroll
          for (int t = 0; t < KC; ++t) { o[h][t][e] *= f; o[h][t][2 + e] *= f; }
        }
    }
    uint32_t hi[NH][2], lo[NH][2];     // P^T as operand: keys 2c, 2c + 1 (and + 8) of head g
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = exp2_approx(s[h][i] - (m[h][i & 1] == -INFINITY ? 0.f : m[h][i & 1]));
      l[h][0] += p[0] + p[2];
      l[h][1] += p[1] + p[3];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t top = pack_bf16(p[2 * i], p[2 * i + 1]);
        hi[h][i] = transpose8x8(top);
        lo[h][i] = transpose8x8(pack_bf16(p[2 * i] - __uint_as_float(top << 16), p[2 * i + 1] - __uint_as_float(top & 0xffff0000u)));
      }
    }
    // V transposed: (channels, keys) (0, 0), (8, 0), (0, 8), (8, 8)
    const uint32_t va = at + kHalf + ((lane & 7) + (lane >> 4 << 3)) * kRowBytes + (((lane >> 3 & 1) ^ turn(lane & 7)) << 4);
#pragma unroll
    for (int t = 0; t < KC; ++t) {
      uint32_t f[4];
      ldmatrix4_trans(f, (va ^ (t % 4 << 5)) + t / 4 * 128);
#pragma unroll
      for (int h = 0; h < NH; ++h) mma16816(o[h][t], f[0], f[1], f[2], f[3], hi[h][0], hi[h][1]);
#pragma unroll
      for (int h = 0; h < NH; ++h) mma16816(o[h][t], f[0], f[1], f[2], f[3], lo[h][0], lo[h][1]);
    }
  }
  // rows, references and sums to shared memory: o[row][channel], then m[row], l[row]
  __device__ __forceinline__ void put(float* rows, float* ms, float* ls) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = h * 8 + 2 * c + e;
        float sum = l[h][e];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (g == 0) { ms[r] = m[h][e]; ls[r] = sum; }
#pragma unroll
        for (int t = 0; t < KC; ++t) {
          rows[Partial<WarpBf16>::at(r, t * 16 + g)] = o[h][t][e];
          rows[Partial<WarpBf16>::at(r, t * 16 + 8 + g)] = o[h][t][2 + e];
        }
      }
  }
  static __device__ __forceinline__ void store4(char* row, int d, const float4& v) {
    *reinterpret_cast<uint2*>(row + d * 2) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  }
};

// ---- fp32 ---------------------------------------------------------------------------------------------------------------
// Plain FMAs (the tensor cores' fp32 sums are not exact to 24 bits).  First product: four lanes per key, each with every fourth
// 16-byte piece of two keys' rows; second: each lane owns four channels of all keys and is sent the weights.
// DC: channels in units of 128; R: query heads
template <int DC, int R>
struct WarpFp32 {
  static constexpr int kRows = R, kWidth = 128 * DC, KC = 8 * DC;
  static constexpr int kStage = kPiece * kWidth * 4 * 2;
  static constexpr int RL = (R + 3) / 4;                     // rows whose weights a lane computes: lane % 4 + 4 i
  static constexpr int kRowBytes = kWidth * 4;
  const unsigned char* qrows;
  float4 o[R][DC];
  float m[R], l[RL];

  static __device__ __forceinline__ uint32_t q_unit(int r, int x) { return r * kRowBytes + x * 16; }
  __device__ __forceinline__ void load_q(const unsigned char* rows) { qrows = rows; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int d = 0; d < DC; ++d) o[r][d] = make_float4(0.f, 0.f, 0.f, 0.f);
      m[r] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < RL; ++i) l[i] = 0.f;
  }
  __device__ __forceinline__ void fetch(const DecodeArgs& a, const Walk& w, uint32_t stage) {
    // 32 units, 128 channels, at a time; wider rows: one half after the other
    const int lane = threadIdx.x & 31;
    const uint32_t dst = stage + lane * 16, k0 = stage + k_lane(0), k1 = stage + k_lane(1);
    // row n of K and V; `at`: bytes from k and v to it, constant
    auto row = [&](auto cn, auto cat, const char* k, const char* v, int bytes) {
      constexpr int n = decltype(cn)::value, at = decltype(cat)::value, odd = n & 1;
      unrolled<DC>([&](auto cd) {
        constexpr int d = decltype(cd)::value;
        const int b = DC == 1 || d * 128 + lane * 4 < a.dh ? bytes : 0;
        copy16<((n / 8) * KC + d * 8) * 512 + (n % 8 - odd) * 64, at + d * 512>(odd ? k1 : k0, k, b);
        copy16<(2 * KC + n * DC + d) * 512, at + d * 512>(dst, v, b);
      });
    };
    if (a.aligned && w.mask == 0xffffu && w.own < 0 && a.dh == kWidth && a.row == kRowBytes / 16) {
      const char *k = w.k + w.off + lane * 16, *v = w.v + w.off + lane * 16;
      unrolled<kPiece>([&](auto cn) { row(cn, Const<decltype(cn)::value * kRowBytes>(), k, v, 16); });
      return;
    }
    const bool there = lane * 4 < a.dh;                      // (of the first 128 channels)
    if (a.near_rows && w.mask == 0xffffu && w.own < 0) {
      const uint32_t units = uint32_t(w.off >> 4);
      unrolled<kPiece>([&](auto cn) {
        constexpr int n = decltype(cn)::value;
        const uint64_t off = uint64_t(a.aligned ? units + n * a.row : __shfl_sync(0xffffffffu, units, n)) * 16 + lane * 16;
        row(cn, Const<0>(), w.k + off, w.v + off, there ? 16 : 0);
      });
      return;
    }
    unrolled<kPiece>([&](auto cn) {
      constexpr int n = decltype(cn)::value;
      const int64_t off = a.aligned ? w.off + bytes_of(n, a.row) : __shfl_sync(0xffffffffu, w.off, n);
      row(cn, Const<0>(), (n == w.own ? w.k_new : w.k + off) + lane * 16, (n == w.own ? w.v_new : w.v + off) + lane * 16,
          there && ((w.mask >> n) & 1) ? 16 : 0);
    });
  }
  __device__ __forceinline__ void use(const DecodeArgs& a, const unsigned char* stage, unsigned mask) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint4* src = reinterpret_cast<const uint4*>(stage);
    float s[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[0][r] = s[1][r] = 0.f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const uint4 u0 = src[kc * 32 + k_slot(kc)], u1 = src[(KC + kc) * 32 + k_slot(kc)];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(qrows + r * kRowBytes + kc * 64 + c * 16);
        s[0][r] = fmaf(__uint_as_float(u0.x), x.x, fmaf(__uint_as_float(u0.y), x.y, fmaf(__uint_as_float(u0.z), x.z, fmaf(__uint_as_float(u0.w), x.w, s[0][r]))));
        s[1][r] = fmaf(__uint_as_float(u1.x), x.x, fmaf(__uint_as_float(u1.y), x.y, fmaf(__uint_as_float(u1.z), x.z, fmaf(__uint_as_float(u1.w), x.w, s[1][r]))));
      }
    }
    bool grows = false;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x = s[i][r];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        x *= a.scale_log2;
        if (!((mask >> (g + i * 8)) & 1)) x = -INFINITY;
        s[i][r] = x;
        grows |= x > m[r] + 8.f;
      }
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = fmaxf(s[0][r], s[1][r]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = fminf(fmaxf(top, m[r]), FLT_MAX);
        const float f = top == -INFINITY ? 1.f : exp2_approx(m[r] - top);
        m[r] = top;
        if ((r & 3) == c) l[r >> 2] *= f;
#pragma unroll
        for (int d = 0; d < DC; ++d) { o[r][d].x *= f; o[r][d].y *= f; o[r][d].z *= f; o[r][d].w *= f; }
      }
    }
    float p[2][RL];
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      float x0 = -INFINITY, x1 = -INFINITY, ref = 0.f;       // row c + 4 i
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * i + e < R && e == c) { x0 = s[0][4 * i + e]; x1 = s[1][4 * i + e]; ref = m[4 * i + e]; }
      if (ref == -INFINITY) ref = 0.f;
      p[0][i] = exp2_approx(x0 - ref);
      p[1][i] = exp2_approx(x1 - ref);
      l[i] += p[0][i] + p[1][i];
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
      uint4 v[DC];
#pragma unroll
      for (int d = 0; d < DC; ++d) v[d] = src[(2 * KC + i * DC + d) * 32 + lane];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float w = __shfl_sync(0xffffffffu, p[i >> 3][r >> 2], (i & 7) * 4 + (r & 3));
#pragma unroll
        for (int d = 0; d < DC; ++d) {
          o[r][d].x = fmaf(w, __uint_as_float(v[d].x), o[r][d].x);
          o[r][d].y = fmaf(w, __uint_as_float(v[d].y), o[r][d].y);
          o[r][d].z = fmaf(w, __uint_as_float(v[d].z), o[r][d].z);
          o[r][d].w = fmaf(w, __uint_as_float(v[d].w), o[r][d].w);
        }
      }
    }
  }
  __device__ __forceinline__ void put(float* rows, float* ms, float* ls) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      float sum = l[i];
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (g == 0 && c + 4 * i < R) ls[c + 4 * i] = sum;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (lane == 0) ms[r] = m[r];
#pragma unroll
      for (int d = 0; d < DC; ++d) *reinterpret_cast<float4*>(rows + Partial<WarpFp32>::at(r, d * 128 + lane * 4)) = o[r][d];
    }
  }
  static __device__ __forceinline__ void store4(char* row, int d, const float4& v) { *reinterpret_cast<float4*>(row + d * 4) = v; }
};

__device__ __forceinline__ void axpy(float4& acc, float w, const float4& v) {
  acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
}
// weight of a part with reference m where the largest is `top`
__device__ __forceinline__ float part_weight(float m, float top) { return top == -INFINITY ? 0.f : exp2_approx(m - top); }

// A warp's ring and the pieces it walks, those of its Walk below `end`.  start() sends the first copies on their way, run()
// uses the pieces; between the two, and behind run(), the stage at `to` is free.
template <typename W, int NS>
struct Ring {
  unsigned char* base;
  int n_pieces, to, from;
  unsigned masks[NS];                  // keys that count, of the stages in flight, oldest first

  __device__ __forceinline__ void fetch(const DecodeArgs& a, W& acc, Walk& w, int i, unsigned& mask) {
    mask = 0;
    if (i < n_pieces) {
      w.locate(a, i);
      acc.fetch(a, w, smem_u32(base) + to * W::kStage);
      mask = w.mask;
      to = to + 1 == NS ? 0 : to + 1;
    }
    tc::cp_async_commit();
  }
  __device__ __forceinline__ void start(const DecodeArgs& a, W& acc, Walk& w, int end) {
    n_pieces = w.first < end ? unsigned(end - w.first + w.step - 1) / unsigned(w.step) : 0;
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) fetch(a, acc, w, i, masks[i]);
  }
  // `late` is called once, when the last copies are about to be sent
  template <typename F>
  __device__ __forceinline__ void run(const DecodeArgs& a, W& acc, Walk& w, F late) {
    const int call_at = max(n_pieces - NS, 0);
    if (n_pieces == 0) late();
    for (int i = 0; i < n_pieces; ++i) {
      if (i == call_at) late();
      tc::cp_async_wait<NS - 2>();
      __syncwarp();                    // all lanes' copies are there, and the stage before is free
      fetch(a, acc, w, i + NS - 1, masks[NS - 1]);
      if (masks[0]) acc.use(a, base + from * W::kStage, masks[0]);
      from = from + 1 == NS ? 0 : from + 1;
#pragma unroll
      for (int j = 0; j < NS - 1; ++j) masks[j] = masks[j + 1];
    }
    __syncwarp();
  }
};

// the token's own rows into the cache
__device__ __forceinline__ void write_own(const DecodeArgs& a, const Walk& w, int bytes) {
  const unsigned key = w.n - 1;
  int64_t off;
  if (w.table) {
    const unsigned block = Walk::block_of(a, key);
    const int page = w.table[block];
    if (unsigned(page) >= unsigned(a.n_pages)) return;
    off = bytes_of(page, a.page) + bytes_of(key - block * unsigned(a.page_size), a.row);
  } else {
    off = bytes_of(key, a.row);
  }
  for (int i = (threadIdx.x & 31) * 16; i < bytes; i += 512) {
    *reinterpret_cast<uint4*>(const_cast<char*>(w.k) + off + i) = *reinterpret_cast<const uint4*>(w.k_new + i);
    *reinterpret_cast<uint4*>(const_cast<char*>(w.v) + off + i) = *reinterpret_cast<const uint4*>(w.v_new + i);
  }
}

// the query rows of a (request, head, row block) on their way to shared memory; units behind a row and rows behind the last are zero
template <typename W, int THREADS>
__device__ __forceinline__ void copy_q(const DecodeArgs& a, unsigned char* to, int b, int head0, int n_rows) {
  constexpr int CH = W::kRowBytes / 16, EL = W::kRowBytes / W::kWidth;
  const char* rows = a.q + bytes_of(b, a.q_batch) + bytes_of(head0, a.q_head);
#pragma unroll
  for (int u = threadIdx.x; u < W::kRows * CH; u += THREADS) {
    const int r = u / CH, x = u % CH;
    copy16<0, 0>(smem_u32(to) + W::q_unit(r, x), rows + (r < n_rows ? bytes_of(r, a.q_head) : 0) + x * 16, r < n_rows && x * 16 < a.dh * EL ? 16 : 0);
  }
  tc::cp_async_commit();
}

// where the warps of a CTA leave their partial rows (bytes into its shared memory), references and sums
template <typename W, int WARPS>
struct Meeting {
  int at[WARPS];
  float m[WARPS][W::kRows], l[WARPS][W::kRows];
};
// row r, channels d .. d + 3 of all warps
template <typename W, int WARPS>
__device__ __forceinline__ float4 join_warps(const unsigned char* smem, const Meeting<W, WARPS>& meet, int r, int d, float& top, float& sum) {
  top = meet.m[0][r];
  sum = 0.f;
#pragma unroll
  for (int i = 1; i < WARPS; ++i) top = fmaxf(top, meet.m[i][r]);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    const float f = part_weight(meet.m[i][r], top);
    sum = fmaf(f, meet.l[i][r], sum);
    axpy(o, f, *reinterpret_cast<const float4*>(smem + meet.at[i] + Partial<W>::at(r, d) * 4));
  }
  return o;
}
template <typename W>
__device__ __forceinline__ void store_row(const DecodeArgs& a, int b, int head, int d, float4 o, float top, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
  W::store4(a.out + bytes_of(b, a.out_batch) + bytes_of(head, a.out_head), d, o);
  if (d == 0 && a.lse) a.lse[b * a.lse_batch + head * a.lse_head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) / kLog2e;
}
__device__ __forceinline__ void report(const DecodeArgs& a, bool bad, bool cut) {
  if (!a.status) return;
  bad = __any_sync(0xffffffffu, bad);
  cut = __any_sync(0xffffffffu, cut);
  if ((threadIdx.x & 31) == 0 && (bad || cut)) atomicOr(a.status, (bad ? LIGHTKV_STATUS_PAGE : 0u) | (cut ? LIGHTKV_STATUS_COUNT : 0u));
}
template <typename W> __host__ __device__ constexpr int row_bytes(int dh) { return dh * (W::kRowBytes / W::kWidth); }
template <typename W> __host__ __device__ constexpr int q_bytes() { return W::kRows * W::kRowBytes; }

// room for the quads that a CTA of a cluster gets from its peers, times the cluster's size: rounds of the output, each of
// 32 quads per CTA, rounded up
template <typename W> __host__ __device__ constexpr int part_quads() {
  return W::kRows * W::kWidth / 4 + 32 * kMaxCluster;
}

// One cluster per (request, key head, block of query heads): its warps take the pieces in turn; their parts meet in shared
// memory.  Each CTA of a cluster finishes its share of the output: the others send it their parts of that.
template <typename W, int WARPS, int NS, int PER_SM>
__global__ void __launch_bounds__(32 * WARPS, PER_SM) decode_cluster_kernel(const __grid_constant__ DecodeArgs a, int cluster) {
  // the warps' rings | query rows | parts of the cluster's CTAs: rows, references, sums
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int THREADS = 32 * WARPS, kRings = WARPS * NS * W::kStage, QUADS = W::kWidth / 4;
  __shared__ Meeting<W, WARPS> meet;
  grid_dependency_sync();
  const int warp = threadIdx.x >> 5;
  const int rank = cluster > 1 ? (int)tc::cluster_ctarank() : 0;
  const int unit = blockIdx.x / unsigned(cluster);
  const int per_b = a.n_kv_heads * a.row_blocks, b = unit / unsigned(per_b), head = unit - b * per_b;
  const int hk = a.row_blocks == 1 ? head : head / a.row_blocks, rb = head - hk * a.row_blocks;
  const int first = rank * WARPS + warp, step = cluster * WARPS;
  Walk w;
  w.start(a, b, hk, first, step);
  w.look(a, a.cap);                    // in flight beside the number of keys
  const int asked = a.n_keys[b];
  w.look_slot(a, b);
  const int head0 = hk * a.group + rb * W::kRows, n_rows = min(W::kRows, a.group - rb * W::kRows);
  copy_q<W, THREADS>(a, smem + kRings, b, head0, n_rows);
  if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // all CTAs of the cluster run
  w.n = min(max(asked, 0), a.cap);
  W acc;
  Ring<W, NS> ring;
  ring.base = smem + warp * (NS * W::kStage);
  ring.to = ring.from = 0;
  ring.start(a, acc, w, (int)((unsigned(w.n) + kPiece - 1) / kPiece));
  tc::cp_async_wait<NS - 1>();
  __syncthreads();                     // the query rows are there
  acc.load_q(smem + kRings);
  acc.clear();
  ring.run(a, acc, w, [] {});
  if (rb == 0 && w.k_new && w.n > 0 && unsigned(w.n - 1) / kPiece % step == first) write_own(a, w, row_bytes<W>(a.dh));
  report(a, w.bad, warp == 0 && asked > w.n);

  static_assert(Partial<W>::kBytes <= W::kStage, "a stage holds a warp's partial rows");
  unsigned char* mine = ring.base + ring.to * W::kStage;
  if ((threadIdx.x & 31) == 0) meet.at[warp] = int(mine - smem);
  acc.put(reinterpret_cast<float*>(mine), meet.m[warp], meet.l[warp]);
  if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  // every 32 quads of the output are finished by another CTA, in whose shared memory lie the parts of quad u from all of them
  const uint32_t parts = smem_u32(smem + kRings + q_bytes<W>());
  const int n_quads = n_rows * QUADS;
  for (int u = threadIdx.x; u < n_quads; u += THREADS) {
    const int r = u / QUADS, d = u % QUADS * 4;
    float top, sum;
    const float4 o = join_warps<W, WARPS>(smem, meet, r, d, top, sum);
    if (cluster == 1) {
      if (d < a.dh) store_row<W>(a, b, head0 + r, d, o, top, sum);
    } else {
      const int owner = u / 32 % cluster;
      const uint32_t at = tc::map_to_cta(parts + ((u / 32 / cluster * 32 + u % 32) * cluster + rank) * 16, owner);
      const uint32_t ml = tc::map_to_cta(parts + part_quads<W>() * 16 + (r * cluster + rank) * 8, owner);
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(o.x), "f"(o.y), "f"(o.z), "f"(o.w) : "memory");
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(ml), "f"(top), "f"(sum) : "memory");
    }
  }
  if (cluster == 1) return;
  cluster_sync();
  const float4* rows = reinterpret_cast<const float4*>(smem + kRings + q_bytes<W>());
  const float2* sums = reinterpret_cast<const float2*>(rows + part_quads<W>());
  for (int j = warp; (j * cluster + rank) * 32 < n_quads; j += WARPS) {
    const int u = (j * cluster + rank) * 32 + threadIdx.x % 32, r = u / QUADS, d = u % QUADS * 4;
    if (u >= n_quads) break;
    float top = sums[r * cluster].x, sum = 0.f;
    for (int i = 1; i < cluster; ++i) top = fmaxf(top, sums[r * cluster + i].x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < cluster; ++i) {
      const float2 ml = sums[r * cluster + i];
      const float f = part_weight(ml.x, top);
      sum = fmaf(f, ml.y, sum);
      axpy(o, f, rows[(j * 32 + threadIdx.x % 32) * cluster + i]);
    }
    if (d < a.dh) store_row<W>(a, b, head0 + r, d, o, top, sum);
  }
}

// ---- items ----------------------------------------------------------------------------------------------------------------
// A request's keys are cut into equal parts of about total / MOST blocks of kPiece keys per warp (MOST: kItemsPerSlot for each CTA
// that fits on the SMs), one item per part, key head and row block.  CTAs take items as they become free: a resident CTA cancels
// the launch of one that has not started and does its work.  (Fixed equal shares of all keys, cut wherever they end, 132 against
// 95 us for 96 requests of 37 to 8192 keys: shares of many short requests take longer.)  The parts of a request that was cut go to
// the workspace and are joined by decode_join_kernel.
constexpr int kItemsPerSlot = 2;
constexpr int kMinBlocks = 4;         // of a part

template <typename W> __host__ __device__ constexpr int part_floats() { return (W::kRows * (W::kWidth + 2) + 3) / 4 * 4; }   // rows on 16 bytes
// With n blocks in all and parts of c > n / most, fewer than `most` requests are cut (heads and row blocks counted apart), into fewer
// than 2 `most` parts, and there are fewer than `most` items more than requests.
template <typename W> constexpr size_t items_bytes(int most) {
  return sizeof(JoinHeader) + (size_t(most) * sizeof(JoinRecord) + 255) / 256 * 256 + size_t(most) * 2 * part_floats<W>() * 4;
}

template <typename W, int WARPS, int NS, int PER_SM>
__global__ void __launch_bounds__(32 * WARPS, PER_SM) decode_items_kernel(const __grid_constant__ DecodeArgs a, int batch, double inv_parts, JoinHeader* header,
                                                                         JoinRecord* records, float* parts) {
  // the warps' rings | query rows of this item and the next
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int THREADS = 32 * WARPS, kBlock = kPiece * WARPS, kRings = WARPS * NS * W::kStage, QUADS = W::kWidth / 4;
  __shared__ unsigned warp_blocks[WARPS];
  __shared__ int warp_sums[3][WARPS];
  __shared__ int items_at[THREADS + 1], slots_at[THREADS], splits_at[THREADS + 1], keys_at[THREADS];   // per run of requests
  __shared__ Meeting<W, WARPS> meet;
  __shared__ __align__(16) unsigned char answer[16];
  __shared__ __align__(8) uint64_t answered;
  __shared__ int abort_flag;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  if (t == 0) {
    tc::mbar_init(&answered, 1);
    tc::fence_barrier_init();
    abort_flag = 0;
  }
  grid_dependency_sync();
  const int heads = a.n_kv_heads * a.row_blocks;
  auto keys_of = [&](int b) { return min(max(a.n_keys[b], 0), a.cap); };
  auto blocks_of = [&](int n) { return (unsigned(n) + kBlock - 1) / kBlock; };

  // all blocks (the host has seen to it that they are counted in 32 bits); each thread looks at a run of requests
  const int run = unsigned(batch + THREADS - 1) / THREADS, b_lo = min(t * run, batch), b_hi = min(b_lo + run, batch);
  unsigned blocks = 0;
  int n0 = 0;
  for (int b = b_lo; b < b_hi; ++b) blocks += blocks_of(n0 = keys_of(b));
  keys_at[t] = n0;                     // of use where a run is one request
  {
    // sums of 16 bits each, so that a warp's fit 32
    const unsigned lo = __reduce_add_sync(0xffffffffu, blocks & 0xffffu), hi = __reduce_add_sync(0xffffffffu, blocks >> 16);
    if (lane == 0) warp_blocks[warp] = (hi << 16) + lo;
  }
  __syncthreads();
  unsigned total = 0;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) total += warp_blocks[i];
  const unsigned chunk = max(unsigned(kMinBlocks), unsigned(double((unsigned long long)total * heads) * inv_parts) + 1u);
  auto parts_of = [&](int n) { return n > 0 ? (blocks_of(n) + chunk - 1) / chunk : 1u; };
  // items, slots of cut requests and cut requests in front of the run
  int sums[3] = {0, 0, 0};
  for (int b = b_lo; b < b_hi; ++b) {
    const int p = parts_of(run == 1 ? n0 : keys_of(b));
    sums[0] += p * heads;
    if (p > 1) { sums[1] += p * heads; sums[2] += heads; }
  }
  int upto[3] = {sums[0], sums[1], sums[2]};
#pragma unroll
  for (int d = 1; d < 32; d <<= 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int o = __shfl_up_sync(0xffffffffu, upto[i], d);
      if (lane >= d) upto[i] += o;
    }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (lane == 31) warp_sums[i][warp] = upto[i];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < WARPS; ++j)
#pragma unroll
    for (int i = 0; i < 3; ++i) upto[i] += j < warp ? warp_sums[i][j] : 0;
  items_at[t + 1] = upto[0];
  if (t == 0) items_at[0] = 0;
  slots_at[t] = upto[1] - sums[1];
  splits_at[t] = upto[2] - sums[2];
  if (t == THREADS - 1) splits_at[THREADS] = upto[2];
  __syncthreads();
  const int n_items = items_at[THREADS];
  if (int(blockIdx.x) >= n_items) return;

  struct Item { int b, n, parts, part, slot, record, head0, n_rows; };
  static_assert(Partial<W>::kBytes <= W::kStage, "a stage holds a warp's partial rows");
  bool bad = false, cut = false, lost = false;
  uint32_t parity = 0;
  Walk w;
  W acc;
  Ring<W, NS> ring;
  ring.base = smem + warp * (NS * W::kStage);
  ring.to = ring.from = 0;
  Item it = {};
  int item = blockIdx.x;
  for (int q_at = 0;; q_at ^= 1) {     // (the first time round nothing is under way yet)
    const Item now = it;
    const bool open = now.parts > 0;
    bool heard = true;
    if (open) {
      acc.load_q(smem + kRings + (q_at ^ 1) * q_bytes<W>());
      acc.clear();
      ring.run(a, acc, w, [&] {        // which item comes next: asked late, so that no CTA sits on one that others could start
        if (t == 0) {
          tc::mbar_expect_tx(&answered, 16);
          tc::clc_try_cancel(answer, &answered);
        }
      });
      bad |= w.bad;
      // each thread has its own limit: a warp agrees before its lanes shuffle, the CTA below (warps that heard have sent copies by then)
      heard = __all_sync(0xffffffffu, tc::mbar_wait(&answered, parity, &abort_flag));
      parity ^= 1;
      item = heard ? tc::clc_canceled_cta(answer) : -1;
      tc::fence_proxy_async();         // the answer has been read before the next one is written
      if (!heard && a.status) atomicOr(a.status, LIGHTKV_STATUS_TIMEOUT);
    }
    // the next item's copies are sent on their way before the parts of this one meet
    const bool more = item >= 0 && item < n_items;
    if (more) {
      // by whoever has the first item: CTA 0 may have been cancelled before it started, like any other
      if (item == 0 && t == 0) header->n = splits_at[THREADS];
      int r = 0;
#pragma unroll
      for (int d = THREADS / 2; d; d >>= 1)
        if (items_at[r + d] <= item) r += d;
      it.b = r * run; it.n = run == 1 ? keys_at[r] : keys_of(it.b); it.parts = parts_of(it.n);
      int i = item - items_at[r];
      it.slot = slots_at[r]; it.record = splits_at[r];
      while (i >= it.parts * heads) {  // (runs of several requests)
        i -= it.parts * heads;
        if (it.parts > 1) { it.slot += it.parts * heads; it.record += heads; }
        it.n = keys_of(++it.b);
        it.parts = parts_of(it.n);
      }
      const int head = it.parts == 1 ? i : unsigned(i) / unsigned(it.parts);
      it.part = i - head * it.parts;
      it.slot += i;
      it.record += head;
      const int hk = a.row_blocks == 1 ? head : head / a.row_blocks, rb = head - hk * a.row_blocks;
      it.head0 = hk * a.group + rb * W::kRows;
      it.n_rows = min(W::kRows, a.group - rb * W::kRows);
      const int per = it.parts == 1 ? blocks_of(it.n) : (blocks_of(it.n) + it.parts - 1) / unsigned(it.parts);
      const int first = it.part * per * WARPS + warp, end = min((it.part + 1) * per * WARPS, int((unsigned(it.n) + kPiece - 1) / kPiece));
      w.start(a, it.b, hk, first, WARPS);
      w.n = it.n;
      w.look(a, it.n);
      w.look_slot(a, it.b);
      copy_q<W, THREADS>(a, smem + kRings + q_at * q_bytes<W>(), it.b, it.head0, it.n_rows);
      cut |= it.n == a.cap && a.n_keys[it.b] > it.n;
      const int last = (it.n - 1) / kPiece;
      if (rb == 0 && w.k_new && it.n > 0 && last >= first && last < end && unsigned(last - first) % WARPS == 0) write_own(a, w, row_bytes<W>(a.dh));
      ring.start(a, acc, w, end);
    }
    if (open) {
      unsigned char* own = ring.base + ring.to * W::kStage;
      if (lane == 0) meet.at[warp] = int(own - smem);
      acc.put(reinterpret_cast<float*>(own), meet.m[warp], meet.l[warp]);
      __syncthreads();
      float* mine = parts + size_t(now.slot) * part_floats<W>();
      for (int u = t; u < now.n_rows * QUADS; u += THREADS) {
        const int row = u / QUADS, d = u % QUADS * 4;
        float top, sum;
        const float4 o = join_warps<W, WARPS>(smem, meet, row, d, top, sum);
        if (now.parts == 1) {
          if (d < a.dh) store_row<W>(a, now.b, now.head0 + row, d, o, top, sum);
        } else {
          *reinterpret_cast<float4*>(mine + row * W::kWidth + d) = o;
          if (d == 0) { mine[W::kRows * W::kWidth + row] = top; mine[W::kRows * (W::kWidth + 1) + row] = sum; }
        }
      }
      if (t == 0 && now.parts > 1 && now.part == 0) records[now.record] = {now.b, now.head0, now.parts, now.slot};
    }
    if (more) tc::cp_async_wait<NS - 1>();                   // the query rows are there
    lost = __syncthreads_or(!heard);
    if (lost || !more) break;
  }
  tc::cp_async_wait<0>();
  if (lost && t == 0) {                // the answer is written to this CTA's memory: it gets as long again
    abort_flag = 0;
    tc::mbar_wait(&answered, parity ^ 1, &abort_flag);
  }
  report(a, bad, cut);
}

// The parts of a request that was cut: CTAs take one record after the other and `rows` rows of it; groups of threads take the parts
// in turn.
template <typename W>
__global__ void __launch_bounds__(512) decode_join_kernel(const __grid_constant__ DecodeArgs a, int batch, int most, int rows,
                                                          const JoinHeader* header, const JoinRecord* records, const float* parts) {
  __shared__ float4 os[512];
  __shared__ float tops[512], sums[512];
  constexpr int QUADS = W::kWidth / 4;
  grid_dependency_sync();
  const int n = join_count(header->n, most);
  JoinRecord rec = records[blockIdx.x];                      // (beside the number; behind it: anything)
  for (int i_rec = blockIdx.x; i_rec < n; i_rec += gridDim.x) {
    if (i_rec != int(blockIdx.x)) rec = records[i_rec];
    if (!joinable(rec, batch, a.n_kv_heads * a.group, 2 * most)) continue;
    const int r0 = blockIdx.y * rows, outputs = min(rows, min(W::kRows, a.group - rec.head0 % a.group) - r0) * QUADS;
    const int per_round = min(outputs, 512), groups = outputs > 0 ? 512 / per_round : 0, g = outputs > 0 ? threadIdx.x / per_round : 0;
    const int used = min(groups, rec.parts);
    const float* first = parts + size_t(rec.slot) * part_floats<W>();
    for (int base = 0; base < outputs; base += per_round) {
      const int u = base + threadIdx.x - g * per_round, r = r0 + u / QUADS, d = u % QUADS * 4;
      const bool mine = g < used && u < outputs;
      float top = -INFINITY, sum = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      constexpr int J = 6;
      if (mine)
        for (int i0 = g; i0 < rec.parts; i0 += J * groups) {
          float m[J], l[J];
          float4 x[J];
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const int i = i0 + j * groups;
            m[j] = -INFINITY; l[j] = 0.f; x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < rec.parts) {
              const float* p = first + size_t(i) * part_floats<W>();
              m[j] = p[W::kRows * W::kWidth + r]; l[j] = p[W::kRows * (W::kWidth + 1) + r];
              x[j] = *reinterpret_cast<const float4*>(p + r * W::kWidth + d);
            }
          }
          float next = top;
#pragma unroll
          for (int j = 0; j < J; ++j) next = fmaxf(next, m[j]);
          const float f = part_weight(top, next);
          sum *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
          top = next;
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const float e = part_weight(m[j], top);
            sum = fmaf(e, l[j], sum);
            axpy(o, e, x[j]);
          }
        }
      if (used > 1) {
        os[threadIdx.x] = o; tops[threadIdx.x] = top; sums[threadIdx.x] = sum;
        __syncthreads();
        if (g == 0) {
          const float own = top;
          for (int i = 1; i < used; ++i) top = fmaxf(top, tops[i * per_round + threadIdx.x]);
          const float f = part_weight(own, top);
          sum *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
          for (int i = 1; i < used; ++i) {
            const int at = i * per_round + threadIdx.x;
            const float e = part_weight(tops[at], top);
            sum = fmaf(e, sums[at], sum);
            axpy(o, e, os[at]);
          }
        }
        __syncthreads();
      }
      if (mine && g == 0 && d < a.dh) store_row<W>(a, rec.b, rec.head0 + r, d, o, top, sum);
    }
  }
}

// Shapes of the kernels: warps a CTA, stages of a warp's ring, CTAs per SM that fit.
template <typename W, int WARPS> struct Shape {
  static constexpr int kWarps = WARPS, kStages = W::kStage <= 2048 || (W::kStage <= 4096 && WARPS == 4) ? 6 : 3;
  static constexpr int kRings = kWarps * kStages * W::kStage;
  static constexpr int kPerSm = std::max(1, 227 * 1024 / (kRings + 2 * q_bytes<W>() + 5120));
  static constexpr int kItemsSmem = kRings + 2 * q_bytes<W>();
  static constexpr int kMost = kItemsPerSlot * kPerSm * kSms;
};
template <typename W> using Items = Shape<W, W::kStage <= 16384 ? 4 : 2>;

template <typename W, int WARPS>
cudaError_t launch_clusters(const DecodeArgs& a, long long units, int cluster, cudaStream_t stream) {
  using S = Shape<W, WARPS>;
  auto kernel = decode_cluster_kernel<W, WARPS, S::kStages, S::kPerSm>;
  const int smem = S::kRings + q_bytes<W>() + (cluster > 1 ? part_quads<W>() * 16 + W::kRows * kMaxCluster * 8 : 0);
  const cudaError_t e = ensure_dynamic_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, dim3((unsigned)(units * cluster)), dim3(32 * WARPS), smem, stream, cluster, a, cluster);
}

// Which form a call takes.  Clusters where the longest request that the caller has announced gives a warp at most kLongest pieces
// (rounds): CTAs that fill an SM, as many to a request and head as there are SMs for, up to four waves of CTAs (two where requests are
// short); CTAs of four warps, two on an SM, for more; CTAs of two warps for many requests of up to 256 keys (512, if they are more than
// three to an SM), where a CTA's latency counts and not its bandwidth.  Clusters of eight only where they leave a third of the SMs free: 16 of them did not fit the GPU at once (2 x 600 keys,
// 8 key heads 8.4 us against 5.6 with four).  Items behind that: their plan and the join of their parts take about 6 us, but long requests
// are spread over all SMs.  With few CTAs (under 64 read slower than HBM allows), that pays earlier: a round takes 0.65 us against
// 0.01 us for each of its CTAs at full bandwidth.
// Measured for bf16 heads of 128 and 64 channels with the length of the longest request announced.  The rule is the same for other heads,
// for two blocks of query heads and for fp32, whose rounds hold other amounts.  Where nothing is announced the table's width stands for
// the longest request, and from some width on items are taken whatever the lengths (through the binding, bound given : not given):
// 1 x 404 keys of 32 heads 6.9 : 11.6 us from 32768 tokens on, 16 x 150 .. 1500 13.3 : 18.5 from 8192, 24 x 90 .. 2000 (64) 14.5 : 18.9 from 16384.
//   us a call, bf16, head size 128 (64)       wide         4 warps      items
//   1 x 404 keys, 32 heads                     5.2          6.2          9.4
//   1 x 8000 keys, 8 key heads                 9.8
//   1 x 16000 keys, 4 key heads               14.9                      12.6
//   16 x 150 .. 1500, 8 key heads             13.4         14.3         18.9
//   24 x 90 .. 2000, 8 key heads (64)         12.1         15.1         17.6
//   48 x 301 .. 1399, 40 key heads             122          109          111
//   96 x 0 .. 8192, 8 key heads                 99          113           95
//   64 x 100 .. 800, 8 key heads              22.8         20.0
//   64 x 60 .. 250, 8 key heads               16.0 (two warps: 10.1)
//   61 x 1 .. 77, 8 key heads                 12.1 (two warps: 5.9)
//   2 x 60000 .. 131072, 4 key heads           148          134           73
constexpr int kLongest = 32, kShort = 256;
// the wide CTAs' warps, whose rings fill an SM (24 x 90 .. 2000 keys of 64 channels: eight warps 13.5 us, sixteen 12.1)
template <typename W> constexpr int wide_warps() { return W::kStage <= 4096 ? 16 : 8; }

template <typename W>
cudaError_t launch_form(DecodeArgs a, int batch, int max_keys, void* workspace, cudaStream_t stream) {
  using S = Items<W>;
  a.row_blocks = (a.group + W::kRows - 1) / W::kRows;
  const long long units = (long long)batch * a.n_kv_heads * a.row_blocks;
  // many short requests: CTAs of two warps, of which four share an SM
  if (units > sm_count() && max_keys <= kShort * (units > 3 * sm_count() ? 2 : 1)) return launch_clusters<W, 2>(a, units, 1, stream);
  constexpr bool can_wide = W::kStage <= 8192;               // (rings of eight warps would not fit an SM)
  const bool wide = can_wide && units <= (max_keys <= 1024 ? 2 : 4) * sm_count();
  const int warps = wide ? wide_warps<W>() : S::kWarps, room = (wide ? Shape<W, wide_warps<W>()>::kPerSm : S::kPerSm) * sm_count();
  int cluster = 1;
  while (cluster < kMaxCluster && units * cluster * 2 <= (cluster < 4 ? room : room * 2 / 3) && cluster * warps * kPiece < max_keys) cluster *= 2;
  const long long ctas = units * cluster, rounds = (max_keys + cluster * warps * kPiece - 1ll) / (cluster * warps * kPiece);
  if (rounds <= kLongest && (ctas >= 64 || rounds * (64 - ctas) <= 350)) {
    if constexpr (can_wide)
      if (wide) return launch_clusters<W, wide_warps<W>()>(a, units, cluster, stream);
    return launch_clusters<W, S::kWarps>(a, units, cluster, stream);
  }
  const int rows = std::min(a.group, W::kRows);
  JoinHeader* header = static_cast<JoinHeader*>(workspace);
  JoinRecord* records = reinterpret_cast<JoinRecord*>(header + 1);
  float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + sizeof(JoinHeader) + (size_t(S::kMost) * sizeof(JoinRecord) + 255) / 256 * 256);
  // Parts of total / kMost blocks make up to one item more per request and head; where these are few, a little larger ones, so that
  // no CTA is left with one item more than the others (75.3 -> 73.2 us for the two requests of the table).
  const double inv_parts = 1.0 / (double)(units <= S::kMost / 4 ? S::kMost - units : S::kMost);
  auto kernel = decode_items_kernel<W, S::kWarps, S::kStages, S::kPerSm>;
  cudaError_t e = ensure_dynamic_smem(kernel, S::kItemsSmem);
  if (e == cudaSuccess)
    e = launch_kernel(kernel, dim3((unsigned)(units + S::kMost)), dim3(32 * S::kWarps), S::kItemsSmem, stream, 1, a, batch, inv_parts, header, records, parts);
  // few requests have many parts each: a CTA joins one row of them
  const int per_cta = units <= 64 ? 1 : rows;
  if (e == cudaSuccess)
    e = launch_kernel(decode_join_kernel<W>, dim3((unsigned)std::min<long long>(units, 2 * kSms), (rows + per_cta - 1) / per_cta), dim3(512), 0, stream, 1,
                      a, batch, S::kMost, per_cta, header, records, parts);
  return e;
}

// f(kernel variant) for a type, group and head size
template <typename F>
auto with_variant(int dtype, int group, int dh, F f) {
  if (dtype == LIGHTKV_BF16) {
    if (group <= 8) return dh <= 32 ? f(WarpBf16<0, 1>()) : dh <= 64 ? f(WarpBf16<1, 1>()) : dh <= 128 ? f(WarpBf16<2, 1>()) : f(WarpBf16<4, 1>());
    return dh <= 32 ? f(WarpBf16<0, 2>()) : dh <= 64 ? f(WarpBf16<1, 2>()) : dh <= 128 ? f(WarpBf16<2, 2>()) : f(WarpBf16<4, 2>());
  }
  if (dh <= 128) return group == 1 ? f(WarpFp32<1, 1>()) : group <= 4 ? f(WarpFp32<1, 4>()) : f(WarpFp32<1, 8>());
  return group == 1 ? f(WarpFp32<2, 1>()) : f(WarpFp32<2, 4>());
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

}  // namespace lkv

using namespace lkv;

extern "C" {

size_t lightkv_decode_workspace(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (batch <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || head_dim <= 0 || head_dim % 8 || head_dim > 256 ||
      (dtype != LIGHTKV_BF16 && dtype != LIGHTKV_FP32))
    return 0;
  return with_variant(dtype, n_q_heads / n_kv_heads, head_dim, [](auto v) {
    using W = decltype(v);
    return items_bytes<W>(Items<W>::kMost);
  });
}

int lightkv_decode_attention(const lightkv_decode_args_t* a) {
  if (!a || a->struct_size != sizeof(lightkv_decode_args_t)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->batch <= 0 || a->n_q_heads <= 0 || a->n_kv_heads <= 0 || a->n_q_heads % a->n_kv_heads || a->head_dim <= 0 ||
      a->head_dim % 8 || (a->dtype != LIGHTKV_BF16 && a->dtype != LIGHTKV_FP32))
    return LIGHTKV_ERR_INVALID_ARG;
  if (a->head_dim > 256) return LIGHTKV_ERR_UNSUPPORTED;
  if ((long long)a->batch * a->n_q_heads > 0x0fffffff) return LIGHTKV_ERR_UNSUPPORTED;      // CTAs of a launch
  if (!a->q || !a->k_cache || !a->v_cache || !a->n_keys || !a->out || !a->workspace) return LIGHTKV_ERR_INVALID_ARG;
  if (!a->k_new != !a->v_new || (a->slot_map && !a->k_new) || !aligned(a->slot_map, 8) || a->page_size < 0 || a->max_keys < 0 || a->key_bound < 0) return LIGHTKV_ERR_INVALID_ARG;
  if (a->page_size > 0 ? !a->block_table || a->max_blocks <= 0 || a->n_pages <= 0 : a->max_keys <= 0) return LIGHTKV_ERR_INVALID_ARG;
  if (!isfinite(a->scale) || a->scale < 0.f) return LIGHTKV_ERR_INVALID_ARG;
  const void* ptrs[6] = {a->q, a->k_cache, a->v_cache, a->out, a->k_new, a->v_new};
  for (const void* p : ptrs) if (!aligned(p, 16)) return LIGHTKV_ERR_INVALID_ARG;
  const int64_t el = a->dtype == LIGHTKV_BF16 ? 2 : 4;
  const int64_t strides[9] = {a->q_batch_stride, a->q_head_stride, a->page_stride, a->head_stride, a->row_stride,
                              a->new_batch_stride, a->new_head_stride, a->out_batch_stride, a->out_head_stride};
  for (int64_t s : strides) {
    if (s < 0 || s * el % 16) return LIGHTKV_ERR_INVALID_ARG;
    if (s * el / 16 > 0xffffffffll) return LIGHTKV_ERR_UNSUPPORTED;                          // strides of 64 GB and more
  }
  if (a->row_stride < a->head_dim || a->q == a->out || (a->k_new && a->k_cache == a->v_cache)) return LIGHTKV_ERR_INVALID_ARG;
  if (!aligned(a->workspace, 256) ||
      a->workspace_bytes < lightkv_decode_workspace(a->batch, a->n_q_heads, a->n_kv_heads, a->head_dim, a->dtype))
    return LIGHTKV_ERR_WORKSPACE;

  DecodeArgs d = {};
  d.q = static_cast<const char*>(a->q);
  d.k = static_cast<const char*>(a->k_cache); d.v = static_cast<const char*>(a->v_cache);
  d.k_new = static_cast<const char*>(a->k_new); d.v_new = static_cast<const char*>(a->v_new);
  d.out = static_cast<char*>(a->out);
  d.lse = a->lse; d.n_keys = a->n_keys; d.status = a->status;
  d.slot_map = reinterpret_cast<const long long*>(a->slot_map);
  d.table = a->page_size > 0 ? a->block_table : nullptr;
  auto units = [&](int64_t stride) { return (uint32_t)(stride * el / 16); };
  d.q_batch = units(a->q_batch_stride); d.q_head = units(a->q_head_stride);
  d.page = units(a->page_stride); d.head = units(a->head_stride); d.row = units(a->row_stride);
  d.new_batch = units(a->new_batch_stride); d.new_head = units(a->new_head_stride);
  d.out_batch = units(a->out_batch_stride); d.out_head = units(a->out_head_stride);
  d.lse_batch = a->lse_batch_stride; d.lse_head = a->lse_head_stride;
  d.n_kv_heads = a->n_kv_heads; d.group = a->n_q_heads / a->n_kv_heads; d.dh = a->head_dim;
  page_divider(a->page_size > 0 ? (unsigned)a->page_size : 1u, &d.page_mul, &d.page_shift);
  d.aligned = a->page_size % kPiece == 0;
  // units from the caches' start to the last row of a head, as the kernels reach it: pages (or rows of a request) and rows in a page
  d.near_rows = ((double)d.page * (a->page_size > 0 ? a->n_pages : 0) + (double)d.row * (a->page_size > 0 ? a->page_size : a->max_keys)) < 4294967296.0;
  d.page_size = a->page_size; d.max_blocks = a->max_blocks; d.n_pages = a->n_pages;
  long long bound = a->page_size > 0 ? (long long)a->max_blocks * a->page_size : a->max_keys;
  if (bound > 0x7fffff00ll) bound = 0x7fffff00ll;                                            // keys are counted in 32 bits
  // and so are the blocks of 32 keys of a batch, and of a request over all heads
  if ((bound / 32 + 1) * std::max(a->batch, a->n_q_heads) > 0x7fffffffll) return LIGHTKV_ERR_UNSUPPORTED;
  d.cap = (int)bound;
  const double scale = a->scale != 0.f ? a->scale : 1.0 / sqrt((double)a->head_dim);
  d.scale_log2 = (float)(scale * 1.4426950408889634);
  const int announced = a->page_size > 0 ? a->max_keys : a->key_bound;
  if (announced > 0 && announced < bound) bound = announced;
  const cudaError_t e = with_variant(a->dtype, d.group, d.dh, [&](auto v) {
    return launch_form<decltype(v)>(d, a->batch, (int)bound, a->workspace, static_cast<cudaStream_t>(a->stream));
  });
  return e == cudaSuccess ? LIGHTKV_OK : LIGHTKV_ERR_CUDA;
}

}  // extern "C"
