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

// ---- bf16 MFMA kernels ------------------------------------------------------------------------------------------------------
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef const __attribute__((address_space(3))) char* lds_char_ptr;

// Tiles of 64 rows x d_head lie in LDS row-major, the 16-byte chunks of a row swizzled (XOR on the chunk's number).  swz_row:
// for reads of one chunk per lane from 32 consecutive rows (the operand that contracts over d_head).  swz_col: for the
// transposing read, whose 16 lanes fetch 4 rows x 32 bytes (the operand that contracts over the rows).  Both depend on row % 16 only.
template <int DH>
__device__ __forceinline__ int swz_row(int r) { return DH == 64 ? ((r >> 1) & 7) : (r & 15); }
template <int DH>
__device__ __forceinline__ int swz_col(int r) { return DH == 64 ? (((r >> 1) & 1) << 1) : ((r & 3) << 1); }

// Byte offset of a lane's transposing reads in a tile under swz_col, columns from 32 dt, K step 0: lane 16 G + p points at row
// 4 g + p / 4 (g = lane / 32; the second read is 8 rows on) and the four columns from 32 dt + 16 (G % 2) + 4 (p % 4), and receives
// column 32 dt + lane % 32 of four rows.
template <int DH>
__device__ __forceinline__ int tr_offset(int lane, int dt) {
  const int p = lane & 15, row = 4 * (lane >> 5) + (p >> 2), c = dt * 4 + ((lane >> 4) & 1) * 2 + ((p & 3) >> 1);
  return row * DH * 2 + ((c ^ swz_col<DH>(row)) << 4) + 8 * (p & 1);
}
// the "A" operand of K step i (rows 16 i .. 16 i + 15) from offsets of its two reads
template <int ROWB>
__device__ __forceinline__ bf16x8 read_tr(lds_char_ptr tile, int off0, int off1, int i) {
  const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(tile + off0 + 16 * i * ROWB));
  const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(tile + off1 + (16 * i + 8) * ROWB));
  return __builtin_bit_cast(bf16x8, v8s{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// the values of lanes l % 32 and l % 32 + 32, without LDS.  (Through an empty asm statement: a maximum of the two would
// otherwise be folded into the first.)
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  unsigned a = r[0], b = r[1];
  asm volatile("" : "+v"(a), "+v"(b));
  lo = __builtin_bit_cast(float, a);
  hi = __builtin_bit_cast(float, b);
}

// bf16, d_head 64 / 128, all pointers 16-byte aligned, strides in eights
hipError_t packed_fwd_bf16(const PackedAttn& a, const PackedQkv<bf16_t>& o, void* out, float* lse, hipStream_t st);

}  // namespace pf
