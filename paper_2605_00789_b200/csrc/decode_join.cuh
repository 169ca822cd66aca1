// What the two kernels of lightkv_decode_attention's second form hand over in the workspace: one record per request and head block
// whose keys were cut into parts.
#pragma once

namespace lkv {

struct JoinRecord { int b, head0, parts, slot; };           // request, first query head, parts, the first one's place among the parts
struct JoinHeader { int n; int pad[63]; };                  // records

// The workspace is never cleared, and a CTA whose wait has run out leaves the records and the count that it was to write as they
// were: anything.  Only what lies inside the outputs and the parts may be joined.
__host__ __device__ inline int join_count(int n, int most) { return n < 0 ? 0 : n < most ? n : most; }
__host__ __device__ inline bool joinable(const JoinRecord& r, int batch, int n_q_heads, int slots) {
  return (unsigned)r.b < (unsigned)batch && (unsigned)r.head0 < (unsigned)n_q_heads && r.parts > 0 && r.parts <= slots && r.slot >= 0 &&
         r.slot <= slots - r.parts;
}

}  // namespace lkv
