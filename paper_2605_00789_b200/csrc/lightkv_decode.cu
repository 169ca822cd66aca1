// Attention of one new token per request over a paged (or contiguous) cache: lightkv_decode_attention.
//
//   out = softmax(scale q K^T) V  per (request, query head),  lse = log sum exp(scale q K^T)
//
// Every key and value is read once and used for two dot products per query head, so the pass is bound by HBM wherever the
// query heads of a key head share the read.  A warp walks its own pieces of 16 keys and keeps the running maximum and sum of
// the softmax; nothing is shared between warps before the end, and nothing between lanes before the dot products: each lane
// copies (cp.async) the 16-byte pieces that it will itself need as MMA fragments into a ring of its own and reads them back,
// without a barrier or a shuffle.
//
// bf16: keys are the rows of the first product (S^T = K Q^T, mma.sync m16n8k16: 16 keys x 8 query heads), channels the rows of
// the second (O^T = V^T P^T).  The order of the channels inside a dot product and of the keys inside a sum is free, so a lane's
// fragments are whole 16-byte pieces of its rows: K rows lane / 4 and lane / 4 + 8, V rows 2 (lane % 4) + {0, 1, 8, 9}, whose
// 16-bit halves are paired up by byte permutes.  P is rounded to two bf16 summands (hi + lo, 16 bits of mantissa): with one
// the rounding of P would be as large as the rounding of the output row.
// tcgen05 would need 64 rows of query heads, or V transposed through shared memory, to save arithmetic that HBM hides.
#include <math.h>

#include "launch.h"

namespace lkv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 32;              // keys whose rows a warp looks up at once, one per lane
constexpr int kPiece = 16;             // keys of a ring stage

struct DecodeArgs {
  const char* q; const char* k; const char* v; const char* k_new; const char* v_new;
  char* out;
  float* lse;
  const int* table;                    // nullptr: contiguous
  const int* n_keys;
  uint32_t* status;
  // strides in bytes (lse: elements)
  int64_t q_batch, q_head, page, head, row, new_batch, new_head, out_batch, out_head, lse_batch, lse_head;
  int n_kv_heads, group, row_blocks, dh, page_size, max_blocks, n_pages;
  long long cap;                       // rows a request has room for
  float scale_log2;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, the first `bytes` of them from global memory, the rest zero
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// What a warp knows of one request and key head.
struct Walk {
  const char *k, *v;                   // the head's row 0 of page 0
  const char *k_new, *v_new;           // rows that stand for key n - 1, or nullptr
  const int* table;
  int n;                               // keys
  int page_no;                         // page of this lane's key of the tile that is looked up next (-1: none)
  int64_t off;                         // bytes to its row, of the tile in hand
  unsigned mask;                       // bit i: key i of the tile in hand is there
  bool bad;                            // a page number outside the pool was met

  // page number of this lane's key of tile t
  __device__ __forceinline__ int page_of(const DecodeArgs& a, int t, int limit) const {
    const unsigned key = unsigned(t) * kTile + (threadIdx.x & 31);
    if (key >= unsigned(limit)) return -1;
    return table ? table[key / unsigned(a.page_size)] : 0;
  }
  // rows of tile t, whose page numbers are in page_no
  __device__ __forceinline__ void locate(const DecodeArgs& a, int t) {
    const unsigned key = unsigned(t) * kTile + (threadIdx.x & 31);
    bool ok = key < unsigned(n);
    if (table) {
      const bool in_pool = unsigned(page_no) < unsigned(a.n_pages);
      bad |= ok && !in_pool;
      ok = ok && in_pool;
      off = ok ? int64_t(page_no) * a.page + int64_t(key % unsigned(a.page_size)) * a.row : 0;
    } else {
      off = ok ? int64_t(key) * a.row : 0;
    }
    mask = __ballot_sync(0xffffffffu, ok);
  }
};

// ---- bf16 ---------------------------------------------------------------------------------------------------------------
// DC: channels in units of 64; NH: query heads in units of 8
template <int DC, int NH>
struct WarpBf16 {
  static constexpr int kRows = 8 * NH, kWidth = 64 * DC, KC = 2 * DC;
  static constexpr int kStage = kPiece * kWidth * 2 * 2;     // bytes: K and V
  uint32_t q[NH][KC][4];
  float o[NH][4 * DC][4];
  float m[NH][2], l[NH][2];            // heads 2 (lane % 4) and the next: reference exponent; this lane's part of the sum

  __device__ __forceinline__ void load_q(const DecodeArgs& a, const char* rows, int n_rows) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (h * 8 + g < n_rows && kc * 32 + c * 8 < a.dh)
          v = *reinterpret_cast<const uint4*>(rows + (h * 8 + g) * a.q_head + kc * 64 + c * 16);
        q[h][kc][0] = v.x; q[h][kc][1] = v.y; q[h][kc][2] = v.z; q[h][kc][3] = v.w;
      }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < NH; ++h) {
#pragma unroll
      for (int t = 0; t < 4 * DC; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[h][t][i] = 0.f;
      m[h][0] = m[h][1] = -INFINITY;
      l[h][0] = l[h][1] = 0.f;
    }
  }
  // copy half `half` of the tile in hand into the stage at `stage`
  __device__ __forceinline__ void fetch(const DecodeArgs& a, const Walk& w, int tile, int half, uint32_t stage) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint32_t dst = stage + lane * 16;
    // the token's own rows, if this half holds them
    const int own = w.k_new ? w.n - 1 - tile * kTile : -1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = half * kPiece + i * 8 + g;
      const int64_t off = __shfl_sync(0xffffffffu, w.off, j);
      const char* src = j == own ? w.k_new : w.k + off;
      const bool ok = (w.mask >> j) & 1;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        copy16(dst + (i * KC + kc) * 512, src + kc * 64 + c * 16, ok && kc * 32 + c * 8 < a.dh ? 16 : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = half * kPiece + 2 * c + (i & 1) + (i >> 1) * 8;
      const int64_t off = __shfl_sync(0xffffffffu, w.off, j);
      const char* src = j == own ? w.v_new : w.v + off;
      const bool ok = (w.mask >> j) & 1;
#pragma unroll
      for (int ch = 0; ch < DC; ++ch)
        copy16(dst + (2 * KC + i * DC + ch) * 512, src + ch * 128 + g * 16, ok && ch * 64 + g * 8 < a.dh ? 16 : 0);
    }
  }
  // 16 keys; bit i of `mask`: key i counts
  __device__ __forceinline__ void use(const DecodeArgs& a, uint32_t stage, unsigned mask) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const uint32_t src = stage + lane * 16;
    float s[NH][4];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[h][i] = 0.f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const uint4 lo = lds16(src + kc * 512), hi = lds16(src + (KC + kc) * 512);
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        mma16816(s[h], lo.x, hi.x, lo.y, hi.y, q[h][kc][0], q[h][kc][1]);
        mma16816(s[h], lo.z, hi.z, lo.w, hi.w, q[h][kc][2], q[h][kc][3]);
      }
    }
    // s[h][0], s[h][1]: key g, heads 2c and 2c + 1; s[h][2], s[h][3]: key g + 8
    bool grows = false;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[h][i] *= a.scale_log2;
        if (mask != 0xffffu && !((mask >> (g + (i >> 1) * 8)) & 1)) s[h][i] = -INFINITY;
        grows |= s[h][i] > m[h][i & 1] + 8.f;
      }
    // The reference of a row is raised only where a logit exceeds it by 2^8: weights stay below 256, sums in range.
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(s[h][e], s[h][2 + e]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          top = fmaxf(top, m[h][e]);
          const float f = top == -INFINITY ? 1.f : exp2_approx(m[h][e] - top);
          m[h][e] = top;
          l[h][e] *= f;
#pragma unroll
          for (int t = 0; t < 4 * DC; ++t) { o[h][t][e] *= f; o[h][t][2 + e] *= f; }
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
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = lds16(src + (2 * KC + i * DC + ch) * 512);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t a0 = __byte_perm(word(v[0], t), word(v[1], t), 0x5410), a1 = __byte_perm(word(v[0], t), word(v[1], t), 0x7632);
        const uint32_t a2 = __byte_perm(word(v[2], t), word(v[3], t), 0x5410), a3 = __byte_perm(word(v[2], t), word(v[3], t), 0x7632);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          mma16816(o[h][ch * 4 + t], a0, a1, a2, a3, hi[h][0], hi[h][1]);
          mma16816(o[h][ch * 4 + t], a0, a1, a2, a3, lo[h][0], lo[h][1]);
        }
      }
    }
  }
  // rows, references and sums to shared memory: o[row][channel], then m[row], l[row]
  __device__ __forceinline__ void put(float* rows, float* ms, float* ls, int stride) {
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
        // channels ch * 64 + g * 8 + 2 t + {0, 1}
#pragma unroll
        for (int ch = 0; ch < DC; ++ch) {
          float4* d = reinterpret_cast<float4*>(rows + r * stride + ch * 64 + g * 8);
          d[0] = make_float4(o[h][ch * 4][e], o[h][ch * 4][2 + e], o[h][ch * 4 + 1][e], o[h][ch * 4 + 1][2 + e]);
          d[1] = make_float4(o[h][ch * 4 + 2][e], o[h][ch * 4 + 2][2 + e], o[h][ch * 4 + 3][e], o[h][ch * 4 + 3][2 + e]);
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
  const char* qrows;
  float4 o[R][DC];
  float m[R], l[RL];
  int n_rows;

  __device__ __forceinline__ void load_q(const DecodeArgs& a, const char* rows, int n) { qrows = rows; n_rows = n; }
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
  __device__ __forceinline__ void fetch(const DecodeArgs& a, const Walk& w, int tile, int half, uint32_t stage) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint32_t dst = stage + lane * 16;
    const int own = w.k_new ? w.n - 1 - tile * kTile : -1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = half * kPiece + i * 8 + g;
      const int64_t off = __shfl_sync(0xffffffffu, w.off, j);
      const char* src = j == own ? w.k_new : w.k + off;
      const bool ok = (w.mask >> j) & 1;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        copy16(dst + (i * KC + kc) * 512, src + kc * 64 + c * 16, ok && kc * 16 + c * 4 < a.dh ? 16 : 0);
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
      const int j = half * kPiece + i;
      const int64_t off = __shfl_sync(0xffffffffu, w.off, j);
      const char* src = j == own ? w.v_new : w.v + off;
      const bool ok = (w.mask >> j) & 1;
#pragma unroll
      for (int d = 0; d < DC; ++d)
        copy16(dst + (2 * KC + i * DC + d) * 512, src + d * 512 + lane * 16, ok && d * 128 + lane * 4 < a.dh ? 16 : 0);
    }
  }
  __device__ __forceinline__ void use(const DecodeArgs& a, uint32_t stage, unsigned mask) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint32_t src = stage + lane * 16;
    float s[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[0][r] = s[1][r] = 0.f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const uint4 u0 = lds16(src + kc * 512), u1 = lds16(src + (KC + kc) * 512);
      const bool there = kc * 16 + c * 4 < a.dh;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        // (the query rows stay in L1: 16 bytes per lane quad)
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (there && r < n_rows) x = *reinterpret_cast<const float4*>(qrows + r * a.q_head + kc * 64 + c * 16);
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
        top = fmaxf(top, m[r]);
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
      for (int d = 0; d < DC; ++d) v[d] = lds16(src + (2 * KC + i * DC + d) * 512);
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
  __device__ __forceinline__ void put(float* rows, float* ms, float* ls, int stride) {
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
      for (int d = 0; d < DC; ++d) *reinterpret_cast<float4*>(rows + r * stride + d * 128 + lane * 4) = o[r][d];
    }
  }
  static __device__ __forceinline__ void store4(char* row, int d, const float4& v) { *reinterpret_cast<float4*>(row + d * 4) = v; }
};

// Partial rows in shared memory: kRows x (kWidth + pad) floats, references, sums.
template <typename W>
struct Partial {
  static constexpr int kStride = W::kWidth + 4;
  static constexpr int kFloats = W::kRows * (kStride + 2);
  static constexpr int kBytes = (kFloats * 4 + 127) / 128 * 128;
  float* base;
  __device__ __forceinline__ float* rows() const { return base; }
  __device__ __forceinline__ float* ms() const { return base + W::kRows * kStride; }
  __device__ __forceinline__ float* ls() const { return base + W::kRows * (kStride + 1); }
};

__device__ __forceinline__ void axpy(float4& acc, float w, const float4& v) {
  acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
}
// weight of a part with reference m where the largest is `top`
__device__ __forceinline__ float part_weight(float m, float top) { return top == -INFINITY ? 0.f : exp2_approx(m - top); }

// A warp's share of a request: tiles first, first + step, ... of its keys.
template <typename W, int NS>
__device__ __forceinline__ void walk_tiles(const DecodeArgs& a, W& acc, Walk& w, int first, int step, int end, uint32_t ring) {
  const int n_pieces = first < end ? 2 * ((end - first + step - 1) / step) : 0;
  unsigned masks[NS];                  // of the stages in flight, oldest first
#pragma unroll
  for (int i = 0; i < NS; ++i) masks[i] = 0;
  int tile = first, half = 0, to = 0, from = 0;
  auto fetch = [&](int i, unsigned& mask) {
    mask = 0;
    if (i < n_pieces) {
      if (half == 0) {
        w.locate(a, tile);
        w.page_no = w.page_of(a, tile + step, w.n);
      }
      acc.fetch(a, w, tile, half, ring + to * W::kStage);
      mask = (w.mask >> (half * kPiece)) & 0xffffu;
      if (half) tile += step;
      half ^= 1;
      to = to + 1 == NS ? 0 : to + 1;
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) fetch(i, masks[i]);
  for (int i = 0; i < n_pieces; ++i) {
    copy_wait<NS - 2>();
    fetch(i + NS - 1, masks[NS - 1]);
    if (masks[0]) acc.use(a, ring + from * W::kStage, masks[0]);
    from = from + 1 == NS ? 0 : from + 1;
#pragma unroll
    for (int j = 0; j < NS - 1; ++j) masks[j] = masks[j + 1];
  }
  copy_wait<0>();
  __syncwarp();                        // the ring is free for all lanes
}

// the token's own rows into the cache
__device__ __forceinline__ void write_own(const DecodeArgs& a, const Walk& w, int bytes) {
  const int key = w.n - 1;
  int page = 0;
  int64_t off = int64_t(key) * a.row;
  if (w.table) {
    page = w.table[key / a.page_size];
    off = int64_t(page) * a.page + int64_t(key % a.page_size) * a.row;
    if (unsigned(page) >= unsigned(a.n_pages)) return;
  }
  for (int i = (threadIdx.x & 31) * 16; i < bytes; i += 512) {
    *reinterpret_cast<uint4*>(const_cast<char*>(w.k) + off + i) = *reinterpret_cast<const uint4*>(w.k_new + i);
    *reinterpret_cast<uint4*>(const_cast<char*>(w.v) + off + i) = *reinterpret_cast<const uint4*>(w.v_new + i);
  }
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t a, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
__device__ __forceinline__ float ld_peer(uint32_t a) { float v; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a)); return v; }
__device__ __forceinline__ float4 ld_peer4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}

// One cluster per (request, key head, block of query heads): its warps take the tiles in turn; their parts meet in shared
// memory, the CTAs' parts in distributed shared memory.
template <typename W, int WARPS, int NS>
__global__ void __launch_bounds__(32 * WARPS) decode_cluster_kernel(const __grid_constant__ DecodeArgs a, int cluster) {
  extern __shared__ __align__(128) unsigned char smem[];
  grid_dependency_sync();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  const int unit = blockIdx.x / cluster;
  const int rb = unit % a.row_blocks, hk = unit / a.row_blocks % a.n_kv_heads, b = unit / a.row_blocks / a.n_kv_heads;
  const int first = rank * WARPS + warp, step = cluster * WARPS;
  Walk w;
  w.table = a.table ? a.table + size_t(b) * a.max_blocks : nullptr;
  w.k = a.k + hk * a.head + (a.table ? 0 : b * a.page);
  w.v = a.v + hk * a.head + (a.table ? 0 : b * a.page);
  w.k_new = a.k_new ? a.k_new + b * a.new_batch + hk * a.new_head : nullptr;
  w.v_new = a.k_new ? a.v_new + b * a.new_batch + hk * a.new_head : nullptr;
  w.bad = false;
  w.page_no = w.page_of(a, first, (int)min(a.cap, 0x7fffffffll));    // in flight beside the number of keys
  const int asked = a.n_keys[b];
  w.n = (int)min((long long)max(asked, 0), a.cap);
  const int head0 = hk * a.group + rb * W::kRows, n_rows = min(W::kRows, a.group - rb * W::kRows);
  W acc;
  acc.load_q(a, a.q + b * a.q_batch + head0 * a.q_head, n_rows);
  acc.clear();
  unsigned char* ring = smem + warp * (NS * W::kStage);
  const int n_tiles = (int)(((long long)w.n + kTile - 1) / kTile);
  walk_tiles<W, NS>(a, acc, w, first, step, n_tiles, smem_addr(ring));
  if (rb == 0 && w.k_new && w.n > 0 && ((w.n - 1) / kTile) % step == first) write_own(a, w, a.dh * (W::kStage / (kPiece * W::kWidth * 2)));
  if (a.status) {
    const bool bad = __any_sync(0xffffffffu, w.bad);
    if (lane == 0 && (bad || (warp == 0 && asked > w.n)))
      atomicOr(a.status, (bad ? LIGHTKV_STATUS_PAGE : 0u) | (asked > w.n ? LIGHTKV_STATUS_COUNT : 0u));
  }

  using P = Partial<W>;
  static_assert(2 * P::kBytes <= NS * W::kStage, "a warp's ring holds its partial rows and the CTA's");
  P mine{reinterpret_cast<float*>(ring)};
  acc.put(mine.rows(), mine.ms(), mine.ls(), P::kStride);
  __syncthreads();
  const int quads = a.dh / 4;
  P cta{reinterpret_cast<float*>(smem + P::kBytes)};         // behind warp 0's part
  auto part = [&](int i) { return P{reinterpret_cast<float*>(smem + i * (NS * W::kStage))}; };
  for (int u = threadIdx.x; u < n_rows * quads; u += 32 * WARPS) {
    const int r = u / quads, d = (u - r * quads) * 4;
    float top = part(0).ms()[r], sum = 0.f;
#pragma unroll
    for (int i = 1; i < WARPS; ++i) top = fmaxf(top, part(i).ms()[r]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
      const float f = part_weight(part(i).ms()[r], top);
      sum = fmaf(f, part(i).ls()[r], sum);
      axpy(o, f, *reinterpret_cast<const float4*>(part(i).rows() + r * P::kStride + d));
    }
    if (cluster == 1) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
      W::store4(a.out + b * a.out_batch + (head0 + r) * a.out_head, d, o);
      if (d == 0 && a.lse) a.lse[b * a.lse_batch + (head0 + r) * a.lse_head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) / kLog2e;
    } else {
      *reinterpret_cast<float4*>(cta.rows() + r * P::kStride + d) = o;
      if (d == 0) { cta.ms()[r] = top; cta.ls()[r] = sum; }
    }
  }
  if (cluster == 1) return;
  cluster_sync();
  for (int u = rank * 32 * WARPS + threadIdx.x; u < n_rows * quads; u += cluster * 32 * WARPS) {
    const int r = u / quads, d = (u - r * quads) * 4;
    const uint32_t am = smem_addr(cta.ms() + r), al = smem_addr(cta.ls() + r), ao = smem_addr(cta.rows() + r * P::kStride + d);
    float top = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float ms[8], ls[8];
    float4 os[8];
    for (int base = 0; base < cluster; base += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (base + i < cluster) {
          ms[i] = ld_peer(peer_addr(am, base + i));
          ls[i] = ld_peer(peer_addr(al, base + i));
          os[i] = ld_peer4(peer_addr(ao, base + i));
        }
      float next = top;
#pragma unroll
      for (int i = 0; i < 8; ++i) if (base + i < cluster) next = fmaxf(next, ms[i]);
      const float f = part_weight(top, next);
      sum *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
      top = next;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (base + i < cluster) {
          const float g = part_weight(ms[i], top);
          sum = fmaf(g, ls[i], sum);
          axpy(o, g, os[i]);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
    W::store4(a.out + b * a.out_batch + (head0 + r) * a.out_head, d, o);
    if (d == 0 && a.lse) a.lse[b * a.lse_batch + (head0 + r) * a.lse_head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) / kLog2e;
  }
  cluster_sync();                      // a CTA's shared memory lives until all have read it
}

template <typename W, int WARPS, int NS>
cudaError_t launch_form(DecodeArgs a, int batch, int max_keys, cudaStream_t stream) {
  a.row_blocks = (a.group + W::kRows - 1) / W::kRows;
  const long long units = (long long)batch * a.n_kv_heads * a.row_blocks;
  int cluster = 1;
  while (cluster < 8 && units * cluster * 2 <= 2 * sm_count() && cluster * WARPS * kTile < max_keys) cluster *= 2;
  constexpr size_t smem = size_t(WARPS) * NS * W::kStage;
  const cudaError_t e = ensure_dynamic_smem(decode_cluster_kernel<W, WARPS, NS>, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(decode_cluster_kernel<W, WARPS, NS>, dim3((unsigned)(units * cluster)), dim3(32 * WARPS), smem, stream, cluster, a, cluster);
}

cudaError_t launch_decode(const DecodeArgs& a, int dtype, int batch, int max_keys, cudaStream_t stream) {
  if (dtype == LIGHTKV_BF16) {
    if (a.group <= 8) {
      if (a.dh <= 64) return launch_form<WarpBf16<1, 1>, 4, 6>(a, batch, max_keys, stream);
      if (a.dh <= 128) return launch_form<WarpBf16<2, 1>, 4, 3>(a, batch, max_keys, stream);
      return launch_form<WarpBf16<4, 1>, 4, 3>(a, batch, max_keys, stream);
    }
    if (a.dh <= 64) return launch_form<WarpBf16<1, 2>, 4, 6>(a, batch, max_keys, stream);
    if (a.dh <= 128) return launch_form<WarpBf16<2, 2>, 4, 3>(a, batch, max_keys, stream);
    return launch_form<WarpBf16<4, 2>, 4, 3>(a, batch, max_keys, stream);
  }
  if (a.dh <= 128) {
    if (a.group == 1) return launch_form<WarpFp32<1, 1>, 4, 3>(a, batch, max_keys, stream);
    if (a.group <= 4) return launch_form<WarpFp32<1, 4>, 4, 3>(a, batch, max_keys, stream);
    return launch_form<WarpFp32<1, 8>, 4, 3>(a, batch, max_keys, stream);
  }
  if (a.group == 1) return launch_form<WarpFp32<2, 1>, 2, 3>(a, batch, max_keys, stream);
  return launch_form<WarpFp32<2, 4>, 2, 3>(a, batch, max_keys, stream);
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
  return 256;
}

int lightkv_decode_attention(const lightkv_decode_args_t* a) {
  if (!a || a->struct_size != sizeof(lightkv_decode_args_t)) return LIGHTKV_ERR_INVALID_ARG;
  if (a->batch <= 0 || a->n_q_heads <= 0 || a->n_kv_heads <= 0 || a->n_q_heads % a->n_kv_heads || a->head_dim <= 0 ||
      a->head_dim % 8 || (a->dtype != LIGHTKV_BF16 && a->dtype != LIGHTKV_FP32))
    return LIGHTKV_ERR_INVALID_ARG;
  if (a->head_dim > 256) return LIGHTKV_ERR_UNSUPPORTED;
  if ((long long)a->batch * a->n_q_heads > 0x0fffffff) return LIGHTKV_ERR_UNSUPPORTED;      // CTAs of a launch
  if (!a->q || !a->k_cache || !a->v_cache || !a->n_keys || !a->out || !a->workspace) return LIGHTKV_ERR_INVALID_ARG;
  if (!a->k_new != !a->v_new || a->page_size < 0 || a->max_keys < 0) return LIGHTKV_ERR_INVALID_ARG;
  if (a->page_size > 0 ? !a->block_table || a->max_blocks <= 0 || a->n_pages <= 0 : a->max_keys <= 0) return LIGHTKV_ERR_INVALID_ARG;
  if (!isfinite(a->scale) || a->scale < 0.f) return LIGHTKV_ERR_INVALID_ARG;
  const void* ptrs[6] = {a->q, a->k_cache, a->v_cache, a->out, a->k_new, a->v_new};
  for (const void* p : ptrs) if (!aligned(p, 16)) return LIGHTKV_ERR_INVALID_ARG;
  const int64_t el = a->dtype == LIGHTKV_BF16 ? 2 : 4;
  const int64_t strides[9] = {a->q_batch_stride, a->q_head_stride, a->page_stride, a->head_stride, a->row_stride,
                              a->new_batch_stride, a->new_head_stride, a->out_batch_stride, a->out_head_stride};
  for (int64_t s : strides) if (s * el % 16) return LIGHTKV_ERR_INVALID_ARG;
  if (a->row_stride < a->head_dim || a->q == a->out) return LIGHTKV_ERR_INVALID_ARG;
  if (!aligned(a->workspace, 256) ||
      a->workspace_bytes < lightkv_decode_workspace(a->batch, a->n_q_heads, a->n_kv_heads, a->head_dim, a->dtype))
    return LIGHTKV_ERR_WORKSPACE;

  DecodeArgs d = {};
  d.q = static_cast<const char*>(a->q);
  d.k = static_cast<const char*>(a->k_cache); d.v = static_cast<const char*>(a->v_cache);
  d.k_new = static_cast<const char*>(a->k_new); d.v_new = static_cast<const char*>(a->v_new);
  d.out = static_cast<char*>(a->out);
  d.lse = a->lse; d.n_keys = a->n_keys; d.status = a->status;
  d.table = a->page_size > 0 ? a->block_table : nullptr;
  d.q_batch = a->q_batch_stride * el; d.q_head = a->q_head_stride * el;
  d.page = a->page_stride * el; d.head = a->head_stride * el; d.row = a->row_stride * el;
  d.new_batch = a->new_batch_stride * el; d.new_head = a->new_head_stride * el;
  d.out_batch = a->out_batch_stride * el; d.out_head = a->out_head_stride * el;
  d.lse_batch = a->lse_batch_stride; d.lse_head = a->lse_head_stride;
  d.n_kv_heads = a->n_kv_heads; d.group = a->n_q_heads / a->n_kv_heads; d.dh = a->head_dim;
  d.page_size = a->page_size; d.max_blocks = a->max_blocks; d.n_pages = a->n_pages;
  d.cap = a->page_size > 0 ? (long long)a->max_blocks * a->page_size : a->max_keys;
  if (d.cap > 0x7fffff00ll) d.cap = 0x7fffff00ll;                                            // keys are counted in 32 bits
  const double scale = a->scale != 0.f ? a->scale : 1.0 / sqrt((double)a->head_dim);
  d.scale_log2 = (float)(scale * 1.4426950408889634);
  long long bound = d.cap;
  if (a->max_keys > 0 && a->max_keys < bound) bound = a->max_keys;
  if (launch_decode(d, a->dtype, a->batch, (int)bound, static_cast<cudaStream_t>(a->stream)) != cudaSuccess) return LIGHTKV_ERR_CUDA;
  return LIGHTKV_OK;
}

}  // extern "C"
