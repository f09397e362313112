// Attention on packed sequences: what its kernels share (internal).
#pragma once

#include "packed.h"
#include "pf_device.h"
#include "pf_kernels.h"

namespace pf {

// Operands of a packed attention call.  Rows of all of them are tokens; head a of Q and out, K/V head a / group of K and V.
template <typename T>
struct PackedQkv {
  const T *q, *k, *v;
  int64_t ld_q, ld_k, ld_v, ld_out;   // elements between rows
  PackedRows rows;
  int32_t h, group, causal;
  float scale;
};

// Keys that query `row` sees: its sequence, up to itself if causal.  An empty span: the row is in no sequence.
__device__ __forceinline__ Span keys_of(const PackedRows& p, int r0, int row, int causal) {
  Span s = packed_span(p, r0, row);
  if (causal && s.lo < s.hi) s.hi = row + 1;
  return s;
}
// Queries that see key `row`
__device__ __forceinline__ Span queries_of(const PackedRows& p, int r0, int row, int causal) {
  Span s = packed_span(p, r0, row);
  if (causal && s.lo < s.hi) s.lo = row;
  return s;
}
// value of lane `lane`, as a scalar
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

constexpr float LN2_P = 0.6931471805599453f;
constexpr float LOG2E_P = 1.4426950408889634f;

// bf16, d_head 64 / 128, operands and strides 16-byte aligned: bf16 MFMAs
hipError_t packed_fwd_bf16(const PackedAttn& a, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st);
hipError_t packed_bwd_bf16(const PackedAttn& a, const void* q, const void* k, const void* v, const void* dout, const float* lse,
                           const float* dsum, void* dq, void* dk, void* dv, float* partial, hipStream_t st);

}  // namespace pf
